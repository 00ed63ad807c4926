// Which places and channels a workgroup of a product in 8-bit integers has.  Nothing but arithmetic and the cross-lane operations of a wave, so
// that tests can run it on the host, with lanes of their own.
//
// Bounds of the experts are data.  Whatever they hold, what is found lies within [0, T) places and [0, E) experts: each bound is clamped before it
// is used, and sums over them, which may pass 32 bits then, are unsigned.
#pragma once

#include <stdint.h>

namespace mq {

struct Block {
    int expert, place, count;  // count = 0: there is no such block
};

// The `block`-th block of BM places, counted expert by expert: no block holds places of two experts.  `bound(e)`: where the places of
// expert e begin, e = 0 .. E.  blocks: how many there are in all.
template <typename Bound>
__device__ __forceinline__ Block find_block(int T, int E, int block, int BM, Bound &&bound, int *blocks = nullptr) {
    // a lane for each expert: blocks up to and with it by a prefix sum
    const int lane = threadIdx.x & 63;
    Block found{0, 0, 0};
    uint32_t before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int e = e0 + lane;
        int lo = 0, hi = 0;
        if (e < E) {
            lo = min(max(bound(e), 0), T);
            hi = min(max(bound(e + 1), lo), T);
        }
        const uint32_t mine = ((uint32_t)(hi - lo) + (uint32_t)BM - 1u) / (uint32_t)BM;
        uint32_t upto = before + mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t v = (uint32_t)__shfl_up((int)upto, o, 64) - before;
            if (lane >= o) upto += v;
        }
        const uint64_t past = __ballot(upto > (uint32_t)block);
        if (past && found.count == 0) {
            // (the expert before has `upto` of at most `block`, which is below 2^31, and no expert has 2^31 blocks: here no sum has wrapped yet)
            const int at = __builtin_ctzll(past), nth = block - __builtin_amdgcn_readlane((int)(upto - mine), at);
            const int place = __builtin_amdgcn_readlane(lo, at) + nth * BM;
            found = Block{e0 + at, place, min(BM, __builtin_amdgcn_readlane(hi, at) - place)};
            if (!blocks) return found;
        }
        before = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
    if (blocks) *blocks = (int)before;
    return found;
}

// A unit of the looped forms: up to UNIT places of one expert and the UNIT channels from n0 on.
struct Unit {
    Block b;
    int n0;
};

// Unit `lid` of tiles_m x tiles_n, tiles_m blocks of places and all tiles of channels for each: four blocks of places at a time, all channels
// for them.  Products by expert: of one expert, whose codes are then read from memory once.
template <int UNIT, typename Bound>
__device__ __forceinline__ Unit unit_at(int lid, int T, int E, bool by_expert, int tiles_m, int tiles_n, Bound &&bound) {
    constexpr int GROUP = 4;
    int first = 0, blocks = tiles_m;   // the expert's
    Block b{0, 0, T};
    if (by_expert) {
        b = find_block(T, E, lid / tiles_n, UNIT, bound);
        if (b.count <= 0) return Unit{b, 0};
        const int lo = min(max(bound(b.expert), 0), T), hi = min(max(bound(b.expert + 1), lo), T);
        first = lid / tiles_n - (b.place - lo) / UNIT;
        blocks = (int)(((uint32_t)(hi - lo) + (uint32_t)UNIT - 1u) / (uint32_t)UNIT);
        b.place = lo;
        b.count = hi - lo;
    }
    const int local = lid - first * tiles_n, width = GROUP * tiles_n;
    const int first_m = local / width * GROUP, gsz = min(blocks - first_m, GROUP);
    const int down = (first_m + local % width % gsz) * UNIT;
    return Unit{Block{b.expert, b.place + down, min(UNIT, b.count - down)}, local % width / gsz * UNIT};
}

// quarter `q` of a unit; its places or its channels may be past the end (count <= 0, n0 >= N)
template <int UNIT>
__device__ __forceinline__ Unit quarter_of(Unit u, int q) {
    const int down = (q & 1) * (UNIT / 2);
    u.b.place += down;
    u.b.count = min(u.b.count - down, UNIT / 2);
    u.n0 += (q >> 1 & 1) * (UNIT / 2);
    return u;
}

}  // namespace mq
