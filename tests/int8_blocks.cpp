// Runs csrc/mq_int8_blocks.h on the host: a wave is 64 contexts that take turns, and meet in every cross-lane operation.  Bounds as the grouping
// writes them: every block and every tile once and none besides, against a plain enumeration.  Bounds as they should not be (descending,
// negative, past the last place, anything): what is found lies within the places, whatever it is.  Built with -fsanitize=undefined: an
// overflow on the way ends the program.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <random>
#include <vector>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;

// ---- a wave --------------------------------------------------------------------------------------------------------------
namespace wave {
constexpr int LANES = 64, STACK = 1 << 16;
ucontext_t main_context, lanes[LANES];
char stacks[LANES][STACK];
int current;
bool done[LANES];
int posted[2][LANES], turn[LANES];
std::function<void()> body;

int meet(int value, const std::function<int(const int *)> &read) {   // leaves a value, waits for the others', reads
    const int lane = current, t = turn[lane]++ & 1;
    posted[t][lane] = value;
    swapcontext(&lanes[lane], &main_context);
    return read(posted[t]);
}
void enter() {
    body();
    done[current] = true;
    swapcontext(&lanes[current], &main_context);
}
void run(std::function<void()> f) {
    body = std::move(f);
    for (int l = 0; l < LANES; ++l) {
        getcontext(&lanes[l]);
        lanes[l].uc_stack.ss_sp = stacks[l];
        lanes[l].uc_stack.ss_size = STACK;
        lanes[l].uc_link = nullptr;
        makecontext(&lanes[l], enter, 0);
        done[l] = false, turn[l] = 0;
    }
    for (bool any = true; any;) {
        any = false;
        for (current = 0; current < LANES; ++current)
            if (!done[current]) swapcontext(&main_context, &lanes[current]), any = true;
    }
}
struct Index {
    struct {
        operator int() const { return current; }
    } x;
} index;
}  // namespace wave

#define threadIdx wave::index
static int __shfl_up(int v, int o, int) {
    const int lane = wave::current;
    return wave::meet(v, [=](const int *p) { return p[lane >= o ? lane - o : lane]; });
}
static uint64_t __ballot(bool v) {
    uint64_t mask = 0;
    wave::meet(v, [&](const int *p) {
        for (int l = 0; l < 64; ++l) mask |= (uint64_t)(p[l] != 0) << l;
        return 0;
    });
    return mask;
}
static int read_lane(int v, int at) {
    return wave::meet(v, [=](const int *p) { return p[at]; });
}
#define __builtin_amdgcn_readlane read_lane

#include "mq_int8_blocks.h"

using namespace mq;

// what a workgroup of the looped forms sees: the number of blocks, clamped as the kernel clamps it
struct Seen {
    Block block;
    int blocks;
    Unit unit, quarters[4];
};
template <int UNIT>
static Seen look(const std::vector<int> &bounds, int T, int block, int lid, int tiles_m, int tiles_n) {
    Seen out[wave::LANES];
    const int E = (int)bounds.size() - 1;
    wave::run([&] {
        Seen &s = out[wave::current];
        auto bound = [&](int e) {
            if (e < 0 || e > E) printf("bound %d of %d asked for\n", e, E), exit(1);
            return bounds[e];
        };
        s.block = find_block(T, E, block, UNIT, bound);
        find_block(T, E, 0, UNIT, bound, &s.blocks);
        s.blocks = min(max(s.blocks, 0), tiles_m);
        s.unit = unit_at<UNIT>(lid, T, E, true, s.blocks, tiles_n, bound);
        for (int q = 0; q < 4; ++q) s.quarters[q] = quarter_of<UNIT>(s.unit, q);
    });
    for (int l = 1; l < wave::LANES; ++l) {   // a wave is of one mind
        const Seen &a = out[0], &b = out[l];
        if (a.block.expert != b.block.expert || a.block.place != b.block.place || a.block.count != b.block.count || a.blocks != b.blocks ||
            a.unit.b.place != b.unit.b.place || a.unit.b.count != b.unit.b.count || a.unit.n0 != b.unit.n0)
            printf("lanes differ\n"), exit(1);
    }
    return out[0];
}

static long checks;
static void need(bool ok, const char *what, const std::vector<int> &bounds, int T, int at) {
    ++checks;
    if (ok) return;
    printf("%s: T %d, at %d, bounds", what, T, at);
    for (size_t i = 0; i < bounds.size() && i < 70; ++i) printf(" %d", bounds[i]);
    printf("\n");
    exit(1);
}

static bool within(const Block &b, int E, int T, int most) {
    return b.count <= 0 || (b.count <= most && b.expert >= 0 && b.expert < E && b.place >= 0 && (int64_t)b.place + b.count <= T);
}

template <int UNIT>
static void ordered(const std::vector<int> &bounds, int T, int tiles_n) {
    const int E = (int)bounds.size() - 1, most = T / UNIT + min(E, T);
    std::vector<Block> want;
    for (int e = 0; e < E; ++e)
        for (int p = bounds[e]; p < bounds[e + 1]; p += UNIT) want.push_back(Block{e, p, min(UNIT, bounds[e + 1] - p)});
    need((int)want.size() <= most, "the bound on blocks", bounds, T, most);
    std::vector<std::vector<int>> times(want.size(), std::vector<int>(tiles_n, 0));
    const int total = (int)want.size() * tiles_n;
    for (int lid = 0; lid < max(total, 1); ++lid) {
        const int block = lid % ((int)want.size() + 3);
        const Seen s = look<UNIT>(bounds, T, block, lid, most, tiles_n);
        need(s.blocks == (int)want.size(), "number of blocks", bounds, T, s.blocks);
        if (block < (int)want.size())
            need(s.block.expert == want[block].expert && s.block.place == want[block].place && s.block.count == want[block].count, "block", bounds, T, block);
        else
            need(s.block.count == 0, "a block past the last", bounds, T, block);
        if (total == 0) break;
        // the tile is one of the blocks, at a whole tile of channels
        size_t i = 0;
        while (i < want.size() && want[i].place != s.unit.b.place) ++i;
        need(i < want.size() && want[i].expert == s.unit.b.expert && want[i].count == s.unit.b.count && s.unit.n0 % UNIT == 0 && s.unit.n0 / UNIT < tiles_n, "tile",
             bounds, T, lid);
        ++times[i][s.unit.n0 / UNIT];
        int places = 0;
        for (int q = 0; q < 4; ++q) {
            const Unit &u = s.quarters[q];
            need(u.n0 == s.unit.n0 + (q >> 1) * UNIT / 2 && u.b.place == s.unit.b.place + (q & 1) * UNIT / 2, "quarter", bounds, T, lid);
            places += max(u.b.count, 0);
        }
        need(places == 2 * s.unit.b.count, "places of the quarters", bounds, T, lid);
    }
    for (auto &row : times)
        for (int n : row) need(n == 1, "every tile once", bounds, T, n);
}

template <int UNIT>
static void anything(const std::vector<int> &bounds, int T, int tiles_n, std::mt19937 &rng) {
    const int E = (int)bounds.size() - 1;
    const int64_t most = (int64_t)T / UNIT + min(E, T);
    const int tiles_m = (int)min<int64_t>(most, 0x7FFFFC00 / tiles_n);
    for (int k = 0; k < 6; ++k) {
        const int block = k == 0 ? 0 : k == 1 ? tiles_m - 1 : (int)(rng() % (uint32_t)tiles_m);
        const int lid = k == 0 ? 0 : k == 1 ? tiles_m * tiles_n - 1 : (int)(rng() % (uint32_t)(tiles_m * tiles_n));
        const Seen s = look<UNIT>(bounds, T, block, lid, tiles_m, tiles_n);
        need(within(s.block, E, T, UNIT), "a block out of the places", bounds, T, block);
        need(within(s.unit.b, E, T, UNIT) && s.unit.n0 >= 0 && s.unit.n0 / UNIT < tiles_n, "a tile out of the places", bounds, T, lid);
        for (const Unit &u : s.quarters) need(within(u.b, E, T, UNIT / 2), "a quarter out of the places", bounds, T, lid);
    }
}

int main() {
    std::mt19937 rng(5);
    auto pick = [&](int n) { return (int)(rng() % (uint32_t)n); };
    for (int E : {1, 2, 3, 40, 63, 64, 65, 130}) {
        for (int k = 0; k < 6; ++k) {
            std::vector<int> bounds{0};
            for (int e = 0; e < E; ++e) bounds.push_back(bounds[e] + (k == 0 ? 0 : pick(3) ? pick(k < 3 ? 3 : 600 / E + 2) : 0));
            const int T = max(1, bounds[E] + (k & 1) * 37);
            ordered<16>(bounds, T, 1);
            ordered<128>(bounds, T, 1 + pick(5));
            ordered<256>(bounds, T, 1 + pick(3));
        }
    }
    for (int E : {1, 2, 8, 64, 65, 1024})
        for (int T : {1, 5, 300, 100000, 0x7FFFFF00})
            for (int kind = 0; kind < 6; ++kind) {
                std::vector<int> bounds(E + 1);
                for (int e = 0; e <= E; ++e)
                    bounds[e] = kind == 0 ? (e & 1 ? T : 0) : kind == 1 ? T - (int)((int64_t)T * e / E) : kind == 2 ? (int)rng() : kind == 3 ? (e & 1 ? 0x7FFFFFFF : (int)0x80000000)
                                : kind == 4 ? pick(T) : (e & 1 ? T + pick(256) : -pick(100));
                anything<16>(bounds, T, 1 + pick(3), rng);
                anything<64>(bounds, T, 1 + pick(9), rng);
                anything<128>(bounds, T, 1 + pick(100), rng);
                anything<256>(bounds, T, 1 + pick(100), rng);
            }
    printf("ok %ld\n", checks);
    return 0;
}
