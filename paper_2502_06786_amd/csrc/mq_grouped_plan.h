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

// Tiles of a wave of the matrix-vector product.  Two tiles share the tokens' way through LDS, which counts for 16 tokens from 8192 rows on (14336 x
// 4096, B = 16: 10.2 us with two, 12.3 with one; 4096 x 14336: 14.4 and 11.8), for up to 4 where memory is kept busy by half as many
// waves (73728 x 4608, B = 1, r = 4: 34.9 and 37.0 us; 28672 x 4096: 13.5 and 13.0), at two bits, which are bound by the vector unit, earlier
// (28672 x 4096: 12.9 and 13.5).  Groups of 32 at four bits leave no registers for it (73728 x 4608: 57 and 51 us).
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
