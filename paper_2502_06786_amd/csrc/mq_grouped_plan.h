// Which forms the products with group scales take (host rules on sizes; host code only, so that tests can ask them without a GPU).
#pragma once

#include <stdint.h>

#include <algorithm>

#include "mq_plan.h"

namespace mq {

// A wave takes tiles of 16 rows and up to 16 tokens, codes in stretches of two pieces (128-byte lines) of a row.
constexpr int kGroupedTokens = 16, kGroupedRows = 16;
constexpr int kHalves = 2, kPieces = 2;  // 64-byte halves of a piece, pieces of a stretch
constexpr int stretch_codes(int r) { return kPieces * kHalves * 512 / r; }

// inputs of a group have to be whole steps of the matrix core and whole pieces of 16 bytes
inline int64_t group_unit(int r) { return r == 2 ? 64 : 32; }
// codes of a chunk: those of half a piece, or as far as groups allow it
inline int chunk_codes(int r, int64_t group) {
    int c = 512 / r;
    while (group % c != 0) c >>= 1;
    return c;
}

// tokens that a wave loads: 4, 8 or 16
constexpr int token_class(int64_t B) { return B <= 4 ? 4 : B <= 8 ? 8 : 16; }

// Tiles of a wave of the matrix-vector product.  Two tiles share the tokens' way through LDS and halve the workgroups.  us with one and two, K = 4096
// (r = 4 and up to 4 tokens: 4608), groups of 128 (r = 8: of 64):
//   16 tokens, r = 4   8192 rows 8.2-8.8, 7.0    12288 10.2, 10.1    28672 19.0, 16.5   (K = 14336, groups of 32, 4096 rows: 11.8, 14.4)
//              r = 2   8192 rows 8.0, 7.7        12288 10.6, 10.6    28672 21.1, 19.1   (4096: 6.6, 7.5)
//              r = 8   8192 rows 11.1, 10.0      12288 15.2, 14.3    28672 36.5, 33.1   (4096: 7.5, 7.7)
//    8 tokens, r = 4   8192 rows 7.2, 6.5        12288 9.1, 8.8      28672 15.6, 14.3;   r = 2   8192 rows 6.9, 6.9   28672 16.2, 15.3
//              r = 8   8192 rows 10.9, 10.0      28672 31.2, 29.3
//     1 token, r = 4   28672 rows 15.3, 19.0     40960 22.4, 23.7    57344 29.8, 28.5    65536 33.3, 32.6    73728 36.0, 35.2
//              r = 2   12288 rows 7.9, 8.9       16384 9.5, 9.2      20480 11.0, 11.1    28672 13.8, 13.7    73728 31.6, 27.6
//              r = 8   8192 rows 10.5, 9.7       16384 16.8, 15.6    28672 28.9, 31.4    73728 64.3, 63.3    (16384, K = 14336: 47.3, 49.3)
//    4 tokens, r = 4   57344 rows 32.7, 30.1     73728 41.6, 37.6
// so at eight bits it is as often a few percent too many as too few up to 4 tokens.  Groups of 32 at four bits leave no registers for it there
// (73728 x 4608: 51 us, 57).
constexpr bool gemv_two_tiles_fit(int r, int chunk, int tokens) { return tokens > 4 || r != 4 || chunk != 32; }
constexpr int gemv_tiles(int r, int chunk, int64_t B, int64_t N) {
    return gemv_two_tiles_fit(r, chunk, token_class(B)) && N >= (B > 4 ? 8192 : r == 4 ? 65536 : 16384) ? 2 : 1;
}

// Tiles of a wave of a layer's products, by the wave tiles (gate, up) and the stretches of them (down) of all experts that may be chosen: two where
// that leaves enough waves (both launches, us).
// gate, up: 16 tokens x 2 of 8, 4096 x 14336, r = 4: 168 us, with one 180; 2 tokens x 4 of 64, 2048 x 768: 13.2 with one, 14.5 with two.
// down: 16 tokens x 2 of 8, 4096 x 14336, r = 4: 168 us, with one 181; one token x 8 of 64, 2048 x 1024: 14.1 with one, 15.7 with two.
constexpr int gate_up_tiles(int64_t F, int64_t experts) { return cdiv(2 * F, 2 * kGroupedRows) * experts >= 2048 ? 2 : 1; }
constexpr int down_tiles(int r, int64_t d, int64_t F, int64_t experts) {
    return cdiv(d, 2 * kGroupedRows) * experts * cdiv(F, stretch_codes(r)) >= 2048 ? 2 : 1;
}

// Workgroups that share the rows of a down product: a workgroup for each compute unit, of as many waves as there are items and room (16 tokens x 4 of
// 128, 2048 x 1408: 50 us, with workgroups of their own rows only 78; x 2 of 8, 4096 x 14336: 168 and 209; one token x 8 of 64, 2048 x 1024: 14.0
// both).
constexpr int kDownSplits = 8;
inline int down_splits(int r, int64_t d, int64_t F, int64_t experts, int tiles) {
    const int64_t items = cdiv(F, stretch_codes(r)) * experts, blocks = cdiv(d, kGroupedRows * tiles);
    return (int)std::max<int64_t>(1, std::min<int64_t>({kDownSplits, 256 / blocks, items / 8}));
}

}  // namespace mq
