// Run on a host by test_stream_plan_cpu.py: how the device cuts keys into pieces, against arithmetic without bounds and against the rules that it stands for.
#include "../paper_2604_20470_amd/csrc/stream_place.h"

#include <cmath>
#include <cstdio>
#include <type_traits>

using namespace dr::stream;
typedef __int128 big;

static uint64_t state = 99;
static uint32_t bits() { state = state * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(state >> 33); }
static int pick(int lo, int hi) { return lo + (int)(((uint64_t)bits() * (uint64_t)((int64_t)hi - lo + 1)) >> 31); }
static int spread(int hi) { const int n = pick(0, 30); return pick(0, hi < (1 << n) ? hi : 1 << n); }
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (round %d)\n", __LINE__, #x, round); return 1; } } while (0)

int main() {
    // whole numbers in, whole numbers out: two kernels that work the same out cannot differ
    static_assert(std::is_same<decltype(piece_chunks(0, 1, 1, 1, 1, 4)), int>::value && std::is_same<decltype(pieces_cost(1, 1, 1)), int64_t>::value &&
                  std::is_same<decltype(tiles_cost(1, 1, 1, 1, 1)), int>::value, "");
    for (int round = 0; round < 400000; ++round) {
        // chunks of 64 sequences, as their lanes add them up
        int64_t all = 0;
        int low = 0, high = 0, longest = 0, tiles_left = (1 << 24) - 1;
        const int sequences = pick(1, 64);
        for (int s = 0; s < sequences; ++s) {
            const int tiles = s + 1 == sequences && !(round & 7) ? tiles_left : pick(0, 1) ? spread(tiles_left) : pick(0, tiles_left < 400 ? tiles_left : 400);
            const int chunks = pick(0, 3) ? spread(1 << 25) : 1 << 25;
            tiles_left -= tiles;
            const int64_t mine = (int64_t)tiles * chunks;
            all += mine;
            CHECK(low_part(mine) >= 0 && high_part(mine) >= 0);
            low += low_part(mine);
            high += high_part(mine);
            CHECK(low >= 0 && high >= 0);
            if (tiles && chunks > longest) longest = chunks;
        }
        CHECK(from_parts(low, high) == all);
        const int budget = 4 * pick(1, 512), splits = pick(1, 64), least = pick(0, 1) ? 4 : 8, waves = 4;
        const int per = piece_chunks(all, budget, longest, splits, least, waves);
        CHECK(per >= least && per % waves == 0 && (big)per * splits >= longest);
        const int coarse = all < (1ll << 31) ? 0 : 64 - 31 - __builtin_clzll((uint64_t)all);           // bits left out
        big want = ((((big)all >> coarse) + budget - 1) / budget) << coarse;
        CHECK(want <= (((big)all + budget - 1) / budget) + ((big)1 << coarse) && want >= ((big)all >> coarse << coarse) / budget);
        if (want > 1000000000) want = 1000000000;
        if (want < ((big)longest + splits - 1) / splits) want = ((big)longest + splits - 1) / splits;
        if (want < least) want = least;
        CHECK(per - want >= 0 && per - want < waves);
        // below 2^24 the same as the quotient in floating point
        if (all < (1 << 24) && longest <= splits * least) CHECK(per == ((int)std::fmax(std::ceil((double)all / budget), least) + waves - 1) / waves * waves);
        // costs: no overflow, and the comparison exact
        const int pieces = spread(1 << 30) + 1, slots = pick(1, 1024), size = per, more = spread(1 << 29) + 1;
        const big c0 = ((big)pieces + slots - 1) / slots * ((big)size + 3), c1 = (((big)pieces / 2 + slots) / slots) * ((big)more + 3);
        if (c0 < ((big)1 << 56) && c1 < ((big)1 << 56)) {
            CHECK(pieces_cost(pieces, slots, size) == (int64_t)c0);
            CHECK(cheaper((int64_t)c1, (int64_t)c0) == (c1 * 100 < c0 * 97));
        }
    }
    // tiles of the last round: the number of pieces that the same rule finds in real numbers, or one that takes as long within the steps
    for (int round = 0; round < 200000; ++round) {
        const int chip = 8 * pick(1, 64), rest = pick(0, chip - 1), longest = spread(1 << 25), splits = pick(1, 64), piece = pick(0, 1) ? 8 : 16, budget = 2 * chip;
        int least = 0x7fffffff, cost[64], chosen = 1;
        double real_least = 1e300, real[64];
        for (int p = 1; p <= 64; ++p) {
            const int time = tiles_cost(longest, p, rest, chip, p > 1 ? piece : 0);
            CHECK(time >= 0);
            const bool fits = time > 0 && (p == 1 || (p <= splits && rest * p <= budget));
            cost[p - 1] = fits ? time : 0x7fffffff;
            real[p - 1] = fits ? (double)((rest * p + chip - 1) / chip) * ((double)longest / p + (p > 1 ? piece : 0)) : 1e300;
            if (cost[p - 1] < least) least = cost[p - 1];
            if (real[p - 1] < real_least) real_least = real[p - 1];
        }
        while (!near_least(cost[chosen - 1], least)) ++chosen;
        CHECK(chosen <= 64);
        if (least == 0x7fffffff) { CHECK(chosen == 1); continue; }
        CHECK(real[chosen - 1] * 0.985 <= real_least || longest < 64);
        for (int p = 1; p < chosen; ++p) CHECK(cost[p - 1] == 0x7fffffff || real[p - 1] > real_least * 1.005);
    }
    std::printf("ok\n");
    return 0;
}
