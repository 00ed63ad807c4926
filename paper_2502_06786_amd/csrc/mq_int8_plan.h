// Which form the product in 8-bit integers takes (host rules on sizes; host code only, so that tests can ask them without a GPU).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "mq_plan.h"

namespace mq {

// FEW: 16 channels x 16 places, operands straight to registers, K over the waves (mq_int8_few.hip).
// MID32, MID64, MID96: 64 channels x 32, 64 or 96 places through LDS, K over workgroups where there are few tiles (mq_int8_mid.hip).
// DEEP128, TILE128, TILE256: tiles that are looped over (mq_int8_tile.hip): of 128 x 128 with four stages in LDS, one workgroup to a compute unit,
// K over workgroups where there are few tiles; of 128 x 128, two workgroups to a compute unit; of 256 x 256.
enum Int8Form { kInt8Few, kInt8Mid32, kInt8Mid64, kInt8Mid96, kInt8Deep128, kInt8Tile128, kInt8Tile256, kInt8Forms };

// What a form costs, in us.  A workgroup's stage of 128 k takes `alone` where it has a compute unit for itself and `full` where `per_cu` of
// them share it; `end` is what a tile costs besides its stages, `launch` what a call does; codes and tokens arrive at `bytes_us` bytes in
// a us at most (the large tiles hold two stages: they wait for memory longer), and ranges of K cost `join` and the traffic of their
// partial sums.  Fitted to 5600 times (13 layers from 6000 x 512 to 28672 x 4096, 1 to 4096 tokens, 1 to 16 ranges; replayed from a graph; root mean
// square of the misfit 5 to 12 %): of the forms and ranges timed at 259 sizes, the one that the rule takes is 2 % slower than the best on
// average, 16 % at worst.
struct Int8Cost {
    int channels, places, per_cu;
    bool looped;
    double launch, end, alone, full, bytes_us, join, join_bytes_us;
};
constexpr Int8Cost kInt8Costs[kInt8Forms] = {
    {16, 16, 3, false, 0.16, 2.89, 0.079, 0.207, 5.3e6, 0, 1},
    {64, 32, 3, false, 2.23, 1.37, 0.183, 0.422, 5.3e6, 2.00, 7.6e6},
    {64, 64, 2, false, 2.50, 1.57, 0.252, 0.459, 5.3e6, 1.57, 7.6e6},
    {64, 96, 2, false, 3.07, 1.58, 0.339, 0.556, 5.3e6, 1.05, 6.7e6},
    {128, 128, 1, true, 2.76, 2.94, 0.319, 0.487, 5.3e6, 1.98, 6.5e6},
    {128, 128, 2, true, 0.0, 3.94, 0.601, 0.823, 3.2e6, 0, 1},
    {256, 256, 1, true, 0.0, 7.57, 1.033, 1.033, 2.25e6, 0, 1},
};
constexpr double kInt8Uneven = 0.7;
constexpr double kInt8TokensUs = 14e6;   // bytes of tokens that the FEW form's workgroups read from the L2s in a us
// Products by expert (105 times of 8 to 64 experts with 8 to 125 tokens each): finding its block costs a workgroup `kInt8FindUs` (one that loops
// over tiles keeps the experts' bounds); codes that few tiles share come late, which a stage feels (`kInt8ExpertStage` times as long), while
// the tiles with two stages get more bytes in a us than from one matrix (`kInt8ExpertBytes` times).  The form taken is 1 % slower than the best on
// average, 12 % at worst.
constexpr double kInt8FindUs = 2.5, kInt8ExpertStage = 1.6, kInt8ExpertBytes = 1.5;

constexpr int64_t kInt8PartBytes = (int64_t)64 << 20;   // partial sums of ranges, at most
constexpr int kInt8MaxSplits = 16;

// bytes of the partial sums of a dense product
inline int64_t int8_part_bytes(const Int8Cost &f, int64_t T, int64_t N, int splits) {
    return splits == 1 ? 0 : cdiv(N, f.channels) * cdiv(T, f.places) * f.channels * f.places * 4 * splits;
}

// A last round of few 256-tiles is done in quarters of 128 x 128 with four stages: in their first round, or two.
constexpr int kInt8QuarterTiles = 128;
constexpr bool int8_quarters(int64_t tiles) { return tiles >= 256 && tiles % 256 != 0 && tiles % 256 <= kInt8QuarterTiles; }
constexpr double kInt8QuarterUs = 1.0;

// T places of E experts (E = 0: a dense product), in blocks of a form.  How many an expert has is not known here: half a block more than
// their share is what sizes that vary cost, on average.
inline double int8_cost(int form, int64_t T, int64_t N, int64_t K, int64_t E, int splits) {
    const Int8Cost &f = kInt8Costs[form];
    const double used = E == 0 ? 1.0 : (double)std::min(E, T);
    const double blocks = E == 0 ? (double)cdiv(T, f.places) : used * std::max(1.0, (double)T / used / f.places + 0.5);
    const double tiles = blocks * (double)cdiv(N, f.channels) * splits, slow = E ? kInt8ExpertStage : 1.0, stages = slow * (double)cdiv(K, 128) / splits;
    double t, rate = f.bytes_us;
    if (f.looped) {
        const double wave = 256.0 * f.per_cu, rounds = (double)(int64_t)(tiles / wave), rest = tiles - rounds * wave;
        // the last round: compute units that share their L2 with fewer others wait less
        double last = rest > 0 ? stages * (rest > 256.0 ? f.full : f.alone) + f.end : 0.0;
        if (form == kInt8Deep128 && rest > 0) last = stages * std::max(f.alone, f.full * rest / 256.0) + f.end;
        if (form == kInt8Tile256 && rounds > 0 && rest > 0 && rest <= kInt8QuarterTiles)
            last = (rest <= 64.0 ? 1.0 : 2.0) * (stages * kInt8Costs[kInt8Deep128].full + kInt8Costs[kInt8Deep128].end) + kInt8QuarterUs;
        t = rounds * (stages * f.full + f.end) + last + (E ? kInt8FindUs : 0.0);
        if (E && form != kInt8Deep128) rate *= kInt8ExpertBytes;
    } else {
        // (some compute units have a workgroup more than their share; with experts the number of tiles is not known that well)
        const double share = tiles / 256.0, most = E ? share : share + kInt8Uneven * (std::ceil(share) - share);
        t = std::max(stages * f.alone, stages * f.full / f.per_cu * most) + (f.end + (E ? kInt8FindUs : 0.0)) * std::max(1.0, share / f.per_cu);
    }
    t = std::max(t, (used * (double)N * (double)K + (double)T * (double)K) / rate);
    if (form == kInt8Few) t += tiles * (double)std::min<int64_t>(T, 16) * (double)K / kInt8TokensUs;
    if (splits > 1) t += f.join + (double)int8_part_bytes(f, T, N, splits) * 2.0 / f.join_bytes_us;
    return f.launch + t;
}

// Workgroups of a form's launch, at most: blocks of one expert hold no places of another.
inline int64_t int8_grid(int form, int64_t T, int64_t N, int64_t E, int splits) {
    const Int8Cost &f = kInt8Costs[form];
    const int64_t blocks = E == 0 ? cdiv(T, f.places) : T / f.places + std::min(E, T);
    return blocks * cdiv(N, f.channels) * splits;
}
// (a launch has less than 2^32 threads)
constexpr int64_t kInt8MostWorkgroups = 0xFFFFFF;   // of 256 threads
constexpr int64_t kInt8MostTiles = 0x7FFFFC00;      // where they are looped over: an id past the last one, up to 512 further, still fits 32 bits

struct Int8Plan {
    int form, splits;
};
// `part_bytes`: room for partial sums
inline Int8Plan make_int8_plan(int64_t T, int64_t N, int64_t K, int64_t E, int64_t part_bytes) {
    Int8Plan best{kInt8Tile256, 1};
    double least = 1e300;
    for (int form = 0; form < kInt8Forms; ++form) {
        const Int8Cost &f = kInt8Costs[form];
        if (!f.looped && int8_grid(form, T, N, E, 1) > kInt8MostWorkgroups) continue;
        const bool cut = E == 0 && form >= kInt8Mid32 && form <= kInt8Deep128;
        for (int s = 1; s <= (cut ? kInt8MaxSplits : 1); ++s) {
            // a range has two stages at least, and only grids of less than four rounds are cut
            if (s > 1 && (cdiv(K, 128) < 2 * s || cdiv(N, f.channels) * cdiv(T, f.places) > 1024 || int8_part_bytes(f, T, N, s) > part_bytes)) break;
            const double t = int8_cost(form, T, N, K, E, s);
            if (t < least) {
                least = t;
                best = Int8Plan{form, s};
            }
        }
    }
    return best;
}

// (calls of 2^45 outputs and more do not)
inline bool int8_launches(const Int8Plan &p, int64_t T, int64_t N, int64_t E) {
    return int8_grid(p.form, T, N, E, p.splits) <= (kInt8Costs[p.form].looped ? kInt8MostTiles : kInt8MostWorkgroups);
}

// Few tokens are quantized by every workgroup of the product for itself (mq_int8_few.hip): one launch instead of two.  A token more in a
// workgroup costs 1.3 us, the launch saved 3 to 5: one token 4096 x 4096 10.7 -> 6.8 us, 4096 x 14336 21.9 -> 15.9, two experts 2304 x 9216 19.7
// -> 15.5; with one matrix four lose (4096 x 4096 10.7 against 9.7 us).  Experts share them out: of 8, 4096 x 4096, six places 26.0 -> 20.4 us, eight 28.8
// -> 27.2, but only where the workgroups are few and four fit a compute unit (18432 x 2304 53 -> 59 us, 2304 x 9216 40 -> 45).
constexpr int kInt8SinglePlaces = 8;                    // in all; an expert may have all of them
constexpr int64_t kInt8SingleK = 16384, kInt8SingleBytes = 131072;   // of a token; of all tokens, in LDS
inline bool int8_single(int64_t T, int64_t N, int64_t K, int64_t E) {
    const int64_t used = E == 0 ? 1 : std::min(E, T), tiles = cdiv(N, 16) * used, bytes = T * (K + 16);
    if (T > kInt8SinglePlaces || T > 3 * used || K > kInt8SingleK || bytes > kInt8SingleBytes || tiles > kInt8MostWorkgroups) return false;
    return T <= 4 || (tiles <= 2048 && bytes <= 40960);
}
// 32 channels to a workgroup instead of 16 where that leaves three workgroups to a compute unit: 28672 x 4096 27.6 -> 26.9 us, 14336 x 4096 16.5
// -> 15.8; below, 4096 x 4096 8.2 -> 9.5.
inline bool int8_single_wide(int64_t T, int64_t N, int64_t E) { return cdiv(N, 16) * (E == 0 ? 1 : std::min(E, T)) >= 768; }

}  // namespace mq
