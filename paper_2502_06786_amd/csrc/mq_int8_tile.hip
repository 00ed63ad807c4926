// The product in 8-bit integers for many tokens: tiles through LDS.  Bound by the matrix core, at the clock that its power allows where the launch is long
// enough for that to show, and by the ends of tiles: 8192 x 28672 x 3584 with a gate 762 us under the counters (2.21 POP/s; the core is busy 61 % of
// the cycles at 1.71 GHz), 2011 x 14336 x 4096 96 us (2.45 POP/s; 54 % at 2.22 GHz, two rounds for 1.75 of tiles).  A tile's operands come through
// LDS once per wave that needs them: 64 x 128 per wave and stage reads 24 KB for 64 products of 16 cycles, 768 of the 2048 clocks for eight waves;
// products with just these reads beside them reach 3.39 POP/s, without 3.56.  A tile's first stage waits for the stores of the tile before too: they are
// counted with the loads and were issued behind them.  What counted:
// stages of 128 k, whose rows are whole lines of the L2 (64 k: 8 % slower); products without a pause, operands of the next half replaced behind
// the last product that uses them; the next tile's first stages on their way, and nothing spilled, while outputs are formed; those through LDS to
// stores of 128 bytes side by side.
#include <algorithm>

#include "mq_int8.h"
#include "mq_linear.h"

namespace mq {

// In place.  The compiler does not see a matrix product here (see mfma16_acc for why and for the waits that are ours then): an operand
// that a vector instruction has written is used two wait states later at the earliest, an accumulator read eight after its product.
__device__ __forceinline__ void mfma_i8_acc(i32x4 &acc, const i32x4 &a, const i32x4 &b) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
}

// A value that the compiler takes for new: what depends on it is formed here and not kept in registers from before a loop.
__device__ __forceinline__ int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// WR x WC waves, each with RB blocks of 16 channels times TB blocks of 16 places; stages of 128 k, NBUF of them in LDS; then the scale,
// zero-point, token scale and token sum of the tile's rows for two tiles, and for each wave 16 rows of outputs.
template <int RB, int TB, int WR, int WC, int NBUF>
struct Int8Tile {
    static constexpr int NW = WR * WC, TN = 16 * RB * WR, TM = 16 * TB * WC;
    static constexpr int STAGE = (TN + TM) * 128;
    static constexpr int PARAMS = NBUF * STAGE, PARAM_SET = (TN + TM) * 8;
    static constexpr int OUT = PARAMS + 2 * PARAM_SET, OS = RB * 32 + 16;   // OS: bytes of a row of outputs
    static constexpr int LDS = OUT + NW * 16 * OS;
};

// Which tiles are taken: `total` of them, `first` counted in units of `unit` places and channels (tiles_m x tiles_n of those in all), each a
// unit, or (QUARTERS) a quarter of one.
struct Int8Tiles {
    int tiles_m, tiles_n, first, total;
};

// Persistent: workgroup i takes tiles i, i + gridDim.x, ...; the first stages of a tile are requested before the outputs of the one
// before are formed.
// CUT: K is cut into ranges whose sums go to ranges.part, as mq_int8_mid.hip leaves them.
template <bool R8, int RB, int TB, int WR, int WC, int NBUF, bool CUT, bool QUARTERS, typename Bound>
__device__ __forceinline__ void int8_tiles(const Int8Args &a, const Int8Tiles &tiles, const Int8Ranges &ranges, uint8_t *smem, Bound &&bound) {
    typedef Int8Tile<RB, TB, WR, WC, NBUF> T;
    typedef __attribute__((address_space(1))) void *global_ptr;
    constexpr int NW = T::NW, CL = T::TN / (8 * NW), XL = T::TM / (8 * NW), LPS = CL + XL, NM = RB * TB;
    static_assert(T::TN % (8 * NW) == 0 && T::TM % (8 * NW) == 0 && T::TN % 64 == 0 && T::TM % 64 == 0 && T::LDS + 4 * (kMaxExperts + 1) <= 160 * 1024, "");
    constexpr int unit = QUARTERS ? 2 * T::TM : T::TM;
    const int tiles_m = tiles.tiles_m, tiles_n = tiles.tiles_n, total = tiles.total;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g4 = lane >> 4, l16 = lane & 15, wr = wave % WR, wc = wave / WR;   // (waves i and i + 4 share a SIMD)

    struct Tile {
        Block b;
        int n0;
        int range;
    };
    const int splits = CUT ? ranges.splits : 1, stages = (a.K + 127) / 128;
    // the first tile from id on, in steps of the grid, that is not empty (quarters may be): id is left at it, or past the last
    auto tile_from = [&](int &id) {
        Tile t = {};
        for (; id < total * splits; id += (int)gridDim.x) {
            const int at = (int)xcd_contiguous_id(id, total * splits), lid = CUT ? at % total : at;
            Unit u = unit_at<unit>(tiles.first + (QUARTERS ? lid / 4 : lid), a.T, a.E, a.offsets != nullptr, tiles_m, tiles_n, bound);
            if (QUARTERS) u = quarter_of<unit>(u, lid & 3);
            t = Tile{u.b, u.n0, CUT ? at / total : 0};
            if (t.b.count > 0 && t.n0 < a.N) break;
        }
        return t;
    };

    uint32_t coff[CL];
    int col;
    bf16_tile_lane<NW>(wave, lane, 0, (uint32_t)a.K, coff[0], col);   // (rows of eight 16-byte chunks as there)
    col *= 2;
#pragma unroll
    for (int i = 1; i < CL; ++i) coff[i] = coff[0] + (uint32_t)(8 * NW * i) * (uint32_t)a.K;
    __amdgpu_buffer_rsrc_t rC, rX;
    uint32_t xoff[XL];
    int k_begin = 0, k_end = a.K;   // of the tile that is being requested

    // Load i of the stage at k0 into buffer `buf`.  INSIDE: the stage lies within the rows; otherwise what stands past their end is
    // requested out of range, which the buffer unit answers with zeros, so that every stage has as many loads in flight.
    auto issue_one = [&](auto inside_tag, int k0, int buf, int i) {
        constexpr bool INSIDE = decltype(inside_tag)::value;
        uint8_t *to = smem + buf * T::STAGE + (wave + i * NW) * 1024;   // (the rows of the tokens follow those of the codes)
        const uint32_t off = i < CL ? coff[i] : xoff[i - CL];
        if constexpr (INSIDE)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(i < CL ? rC : rX, (lds_ptr)to, 16, off, k0, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(i < CL ? rC : rX, (lds_ptr)to, 16, k0 + col < k_end ? off + (uint32_t)k0 : kOOB, 0, 0, 0);
    };
    // The tokens whose rows and parameters this lane requests of a tile: found while the tile before is multiplied.
    static_assert((T::TN + T::TM) / 64 <= NW, "a wave fetches the parameters of 64 rows");
    const bool fetches = wave < (T::TN + T::TM) / 64;
    int tokens[XL], param_row;   // (as they stand in rows; nothing waits for them before begin)
    auto look = [&](const Tile &t) {
        const int lane = here(threadIdx.x & 63);
        const int last = t.b.count - 1;
        param_row = wave < T::TN / 64 ? min(t.n0 + wave * 64 + lane, a.N - 1) : t.b.place + min((wave - T::TN / 64) * 64 + lane, last);
#pragma unroll
        for (int i = 0; i < XL; ++i) tokens[i] = t.b.place + min(wave * 8 + (lane >> 3) + 8 * NW * i, last);
        if (a.rows) {
#pragma unroll
            for (int i = 0; i < XL; ++i) tokens[i] = a.rows[tokens[i]];
            if (fetches && wave >= T::TN / 64) param_row = a.rows[param_row];
        }
    };
    // A tile's parameters (set `set`) and its first two stages.
    auto begin = [&](const Tile &t, int set) {
        if (CUT) {
            k_begin = (int)((int64_t)stages * t.range / splits) * 128;
            k_end = min(a.K, (int)((int64_t)stages * (t.range + 1) / splits) * 128);
        }
        rC = make_rsrc(a.codes + ((int64_t)t.b.expert * a.N + t.n0) * a.K, (uint64_t)(a.N - t.n0) * a.K);
        const int base = a.rows ? 0 : t.b.place;   // (gathered tokens lie within 2 GiB: quantize_and_multiply)
        rX = make_rsrc(a.Xq + (int64_t)base * a.ldq, (uint64_t)(a.M - base) * a.ldq);
#pragma unroll
        for (int i = 0; i < XL; ++i) {   // rows past the block's places: out of range, zeros, which cost neither memory nor much power
            const int row = wave * 8 + (here(lane) >> 3) + 8 * NW * i;
            xoff[i] = row < t.b.count ? (uint32_t)(min(max(tokens[i], 0), a.M - 1) - base) * (uint32_t)a.ldq + (uint32_t)col : kOOB;
        }
        uint8_t *to = smem + T::PARAMS + set * T::PARAM_SET + wave * 512;
        const void *one, *two;
        if (wave < T::TN / 64) {
            const int64_t n = (int64_t)t.b.expert * a.N + param_row;
            one = a.alpha + n, two = a.zero + n;
        } else {
            const int m = min(max(param_row, 0), a.M - 1);
            one = a.scale + m, two = a.sum + m;
        }
        if (fetches) {
            __builtin_amdgcn_global_load_lds((global_ptr)one, (lds_ptr)to, 4, 0, 0);
            __builtin_amdgcn_global_load_lds((global_ptr)two, (lds_ptr)(to + 256), 4, 0, 0);
        }
#pragma unroll
        for (int s = 0; s < NBUF; ++s)
#pragma unroll
            for (int i = 0; i < LPS; ++i) issue_one(std::false_type{}, k_begin + s * 128, s, i);
    };

    // operands of half t of a stage; + 2048 per block of 16 rows
    uint32_t ca[2], xa[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int sw = ((2 * group_chunk(g4) + t) ^ ((l16 >> 1) & 7)) << 4;
        ca[t] = (wr * 16 * RB + l16) * 128 + sw;
        xa[t] = T::TN * 128 + (wc * 16 * TB + l16) * 128 + sw;
    }
    i32x4 acc[RB][TB], wf[2][RB], xf[TB];   // wf: for the two halves of a stage

    // Half t of the stage at k0, which lies in buffer buf: blocks of places one after the other, the operands of a block replaced by those
    // of the next half after its last product.  Half 0 reads the operands of half 1; then the buffer is free, and the loads of the stage
    // after the next go there while half 1 reads the first operands of the next stage.  (The workgroup meets a few products after the
    // last of these reads, not right behind it.)
    auto half = [&](auto inside_tag, auto t_tag, int k0, int buf) {
        constexpr int t = decltype(t_tag)::value;
        const uint8_t *src = smem + (t == 0 ? buf : buf + 1 == NBUF ? 0 : buf + 1) * T::STAGE;
        static_for<NM>([&](auto q_tag) {
            constexpr int q = decltype(q_tag)::value, tb = q / RB, rb = q % RB;
            mfma_i8_acc(acc[rb][tb], wf[t][rb], xf[tb]);
            if constexpr (t == 1 && q == RB - 1) stage_barrier<(NBUF - 2) * LPS, 0>();   // the next stage has landed, every wave has read this one
            if constexpr (rb == RB - 1) xf[tb] = *reinterpret_cast<const i32x4 *>(src + xa[1 - t] + tb * 2048);
            static_for<RB>([&](auto j_tag) {
                constexpr int j = decltype(j_tag)::value;
                if constexpr (q == RB + j * (NM / 2 - RB) / RB) wf[1 - t][j] = *reinterpret_cast<const i32x4 *>(src + ca[1 - t] + j * 2048);
                if constexpr (R8 && q == NM / 2 + 2 + j * (NM / 2 - 5) / RB) {
                    wf[1 - t][j] = signed_codes<R8>(wf[1 - t][j]);
                    asm volatile("" : "+v"(wf[1 - t][j]));   // here and not where it is used
                }
            });
            static_for<t == 1 ? LPS : 0>([&](auto l_tag) {
                constexpr int l = decltype(l_tag)::value;
                if constexpr (q == RB + 1 + l * (NM / 2) / LPS) issue_one(inside_tag, k0 + 128 * NBUF, buf, l);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    // The outputs of a tile, 16 places at a time through LDS that only this wave uses; those of the next 16 are formed while the rows
    // come back.
    auto finish = [&](auto gated_tag, const Tile &t, int set) {
        constexpr bool GATED = decltype(gated_tag)::value;
        constexpr int shift = GATED ? 1 : 0, per = (2 * RB) >> shift, VEC = (16 * per + 63) / 64;   // per: chunks of 8 outputs in a row
        const int lane = here(threadIdx.x & 63), g4 = lane >> 4, l16 = lane & 15;
        const uint8_t *params = smem + T::PARAMS + set * T::PARAM_SET;
        uint8_t *out = smem + T::OUT + wave * 16 * T::OS;
        const int n_out = a.N >> shift, first = (t.n0 + wr * 16 * RB) >> shift;
        const int rows = t.b.count - wc * TB * 16;   // of this wave's places
        const int last = n_out > first && n_out - first < per * 8 ? n_out % 8 : 0;   // outputs past the last whole chunk of the rows, if they are this wave's
        f32x4 ka[RB], kb[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int n = (wr * RB + rb) * 16 + 4 * g4;
            const uint8_t *at = params + (n >> 6) * 512 + (n & 63) * 4;
            channel_factors(*reinterpret_cast<const f32x4 *>(at), *reinterpret_cast<const f32x4 *>(at + 256), a.mult, ka[rb], kb[rb]);
        }
        float scale[TB], sum[TB];
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
            const int row = (wc * TB + tb) * 16 + l16;
            const uint8_t *at = params + T::TN * 8 + (row >> 6) * 512 + (row & 63) * 4;
            scale[tb] = *reinterpret_cast<const float *>(at);
            sum[tb] = (float)*reinterpret_cast<const int32_t *>(at + 256);
        }
        u32x2 o[RB];
        auto form = [&](int tb) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = int8_output<R8>(acc[rb][tb][e], sum[tb], scale[tb], ka[rb][e], kb[rb][e], a.offset);
                if constexpr (GATED)
                    o[rb][0] = pack_bf16x2(gated_value(y[0], y[1], a.gate), gated_value(y[2], y[3], a.gate));
                else
                    o[rb] = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
            }
        };
        auto put = [&]() {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                if constexpr (GATED)
                    *reinterpret_cast<uint32_t *>(out + l16 * T::OS + rb * 16 + 4 * g4) = o[rb][0];
                else
                    *reinterpret_cast<u32x2 *>(out + l16 * T::OS + rb * 32 + 8 * g4) = o[rb];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        uint16_t *y = a.Y + (int64_t)(t.b.place + wc * TB * 16) * n_out + first;
        form(0);
        put();
#pragma unroll
        for (int tb = 0; tb < TB; ++tb, y += 16 * (int64_t)n_out) {
            u32x4 v[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = *reinterpret_cast<const u32x4 *>(out + (i * 64 + lane) / per % 16 * T::OS + (i * 64 + lane) % per * 16);
            if (tb + 1 < TB) form(tb + 1);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int row = (i * 64 + lane) / per, ch = (i * 64 + lane) % per * 8;
                if (row < 16 && tb * 16 + row < rows && first + ch + 8 <= n_out)
                    __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4_any *>(y + (int64_t)row * n_out + ch));
            }
            if (last > 0) {
#pragma unroll 1
                for (int c = lane; c < 16 * 8; c += 64)
                    if (tb * 16 + c / 8 < rows && c % 8 < last)
                        y[(int64_t)(c / 8) * n_out + (n_out - last - first) + c % 8] = *reinterpret_cast<const uint16_t *>(out + c / 8 * T::OS + ((n_out - last - first) + c % 8) * 2);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (tb + 1 < TB) put();
        }
    };

    auto leave = [&](const Tile &t) {   // (of a dense product)
        const int tile = t.n0 / T::TN * tiles_m + t.b.place / T::TM;
        i32x4 *to = ranges.part + ((int64_t)(t.range * total + tile) * NW + wave) * (RB * TB * 64) + lane;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) to[(rb * TB + tb) * 64] = acc[rb][tb];
    };

    int id = blockIdx.x, set = 0;
    Tile cur = tile_from(id);
    if (id >= total * splits) return;
    look(cur);
    begin(cur, set);
    for (;;) {
        int next_id = id + (int)gridDim.x;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = i32x4{0, 0, 0, 0};
        stage_barrier<(NBUF - 1) * LPS, 0>();
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) wf[0][rb] = signed_codes<R8>(*reinterpret_cast<const i32x4 *>(smem + ca[0] + rb * 2048));
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) xf[tb] = *reinterpret_cast<const i32x4 *>(smem + xa[0] + tb * 2048);
        const Tile next = tile_from(next_id);
        if (next_id < total * splits) look(next);
        int k0 = k_begin, buf = 0;
        auto stage = [&](auto inside_tag) {
            half(inside_tag, std::integral_constant<int, 0>{}, k0, buf);
            half(inside_tag, std::integral_constant<int, 1>{}, k0, buf);
            k0 += 128;
            buf = buf + 1 == NBUF ? 0 : buf + 1;
        };
        if (WC > 1 && cur.b.count <= wc * TB * 16) {   // no places for this wave: it only fetches, and leaves its SIMD to the other one.
            // (Both: 8 experts of 1025 tokens, 28672 x 4096, 1070 -> 1036 us; 300 tokens through 14336 x 4096 28.3 -> 27.6)
            for (; k0 < k_end; k0 += 128) {
                stage_barrier<(NBUF - 2) * LPS, 0>();
#pragma unroll
                for (int i = 0; i < LPS; ++i) issue_one(std::false_type{}, k0 + 128 * NBUF, buf, i);
                buf = buf + 1 == NBUF ? 0 : buf + 1;
            }
        }
        while (k0 + 128 * (NBUF + 1) <= k_end) stage(std::true_type{});
        while (k0 < k_end) stage(std::false_type{});
        mfma16_settle();
        stage_barrier<0, 0>();   // the buffers are free
        if (next_id < total * splits) begin(next, 1 - set);
        if (CUT)
            leave(cur);
        else if (a.gate)
            finish(std::true_type{}, cur, set);
        else
            finish(std::false_type{}, cur, set);
        if (next_id >= total * splits) break;
        id = next_id;
        cur = next;
        set = 1 - set;
    }
}

// `tiles_m` blocks of places, or with experts a bound on them.  QUARTERS: a last round of few tiles is done in quarters, with four stages in LDS
// (4100 x 4352 x 4096, 288 tiles: 69.4 us; as a launch of their own with two stages 72.7).
template <bool R8, int RB, int TB, int WR, int WC, int NBUF, int WGS, bool CUT, bool QUARTERS>
__global__ __launch_bounds__(64 * WR * WC, WGS * WR * WC / 4) void int8_tile_kernel(Int8Args a, int tiles_m, int tiles_n, Int8Ranges ranges) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass only needs the launch stub
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    typedef Int8Tile<RB, TB, WR, WC, NBUF> T;
    // The experts' bounds are kept in LDS, and only blocks that exist are counted: a workgroup's share of a bound on their number would leave
    // XCDs idle.
    int32_t *bounds = reinterpret_cast<int32_t *>(smem + T::LDS);
    auto bound = [&](int e) { return bounds[e]; };
    if (a.offsets) {
        for (int e = threadIdx.x; e <= a.E; e += 64 * T::NW) bounds[e] = a.offsets[e];
        __syncthreads();
        int blocks;
        find_block(a.T, a.E, 0, T::TM, bound, &blocks);
        tiles_m = min(max(__builtin_amdgcn_readfirstlane(blocks), 0), tiles_m);
    }
    const int total = tiles_m * tiles_n, rest = total % 256;
    const bool quarters = QUARTERS && int8_quarters(total);
    int8_tiles<R8, RB, TB, WR, WC, NBUF, CUT, false>(a, Int8Tiles{tiles_m, tiles_n, 0, quarters ? total - rest : total}, ranges, smem, bound);
    if constexpr (QUARTERS) {
        typedef Int8Tile<2, 4, 4, 2, 4> Q;
        static_assert(Q::NW == T::NW && 2 * Q::TN == T::TN && 2 * Q::TM == T::TM && Q::LDS <= T::LDS, "");
        if (!quarters) return;
        __syncthreads();   // every wave is done with the rounds' LDS
        int8_tiles<R8, 2, 4, 4, 2, 4, false, true>(a, Int8Tiles{tiles_m, tiles_n, total - rest, 4 * rest}, ranges, smem, bound);
    }
#else
    (void)a;
#endif
}

namespace {

template <bool R8, int RB, int TB, int WR, int WC, int NBUF, int WGS, bool CUT = false>
mq_status launch_tile(const Int8Args &a, Int8Form form, hipStream_t st, const Int8Ranges &ranges = {nullptr, 1}) {
    typedef Int8Tile<RB, TB, WR, WC, NBUF> T;
    static_assert(T::TN == T::TM && (T::TM == 128 || T::TM == 256), "the forms of mq_int8_plan.h");
    const int64_t tiles_n = cdiv(a.N, T::TN), tiles = int8_grid(form, a.T, a.N, a.offsets ? a.E : 0, 1), tiles_m = tiles / tiles_n;
    constexpr auto kernel = int8_tile_kernel<R8, RB, TB, WR, WC, NBUF, WGS, CUT, T::TM == 256>;
    const int lds = T::LDS + (a.offsets ? (a.E + 1) * 4 : 0);
    if (!allow_lds<kernel>(lds)) return MQ_ERR_DEVICE;
    const int64_t most = 256 * WGS;   // workgroups that fit the GPU
    kernel<<<dim3((unsigned)std::min(tiles * ranges.splits, most)), dim3(64 * T::NW), lds, st>>>(a, (int)tiles_m, (int)tiles_n, ranges);
    return launch_status();
}

template <bool R8>
mq_status launch_tiles(const Int8Args &a, Int8Form form, int splits, void *part, hipStream_t st) {
    if (form == kInt8Tile256) return launch_tile<R8, 4, 8, 4, 2, 2, 1>(a, form, st);
    if (form == kInt8Tile128) return launch_tile<R8, 4, 4, 2, 2, 2, 2>(a, form, st);
    if (splits == 1) return launch_tile<R8, 2, 4, 4, 2, 4, 1>(a, form, st);
    const Int8Ranges ranges{static_cast<i32x4 *>(part), splits};
    const mq_status s = launch_tile<R8, 2, 4, 4, 2, 4, 1, true>(a, form, st, ranges);
    return s != MQ_OK ? s : launch_int8_join<2, 4, 4, 2>(a, ranges, st);
}

}  // namespace

mq_status launch_int8_tiles(const Int8Args &a, Int8Form form, int splits, void *part, hipStream_t st) {
    return a.offset != 0.f ? launch_tiles<true>(a, form, splits, part, st) : launch_tiles<false>(a, form, splits, part, st);
}

}  // namespace mq
