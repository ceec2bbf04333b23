// Run on a host by test_norm_plan_cpu.py: the number of pieces against a search of all numbers, and what a search costs.
#include "../paper_2604_20470_amd/csrc/norm_plan.h"

#include <chrono>
#include <cmath>
#include <cstdio>

using namespace dr;

static uint64_t state = 7;
static uint32_t bits() { state = state * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(state >> 33); }
static double unit() { return bits() / 2147483648.0; }
static int64_t spread(double most) { return (int64_t)std::exp(unit() * std::log(most)); }
static double time_of(int64_t runs, int64_t turns, int64_t slots, int64_t n) { return (double)((runs * n + slots - 1) / slots) * (double)((turns + n - 1) / n + 8); }
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (runs %lld, turns %lld, slots %lld: %lld pieces)\n", __LINE__, #x, (long long)runs, (long long)turns, (long long)slots, (long long)got.pieces); return 1; } } while (0)

int main() {
    const int64_t slots_of[] = {256, 304, 512, 768, 1024, 3072, 4096, 200, 240};
    for (int round = 0; round < 6000; ++round) {
        const int64_t slots = slots_of[bits() % 9], runs = spread(round % 5 ? 5000 : 1 << 28), turns = spread(std::fmax(2.0, (double)(1 << 30) / runs));
        const int64_t limit = turns / 4 > 1 ? turns / 4 : 1;
        const NormPieces got = norm_pieces(runs, turns, slots);
        CHECK(got.pieces >= 1 && got.pieces <= limit && (got.pieces == 1 || runs * got.pieces <= 16 * slots));
        CHECK(got.time == time_of(runs, turns, slots, got.pieces));
        double least = time_of(runs, turns, slots, 1);
        for (int64_t n = 2; n <= limit && runs * n <= 16 * slots; ++n) least = std::fmin(least, time_of(runs, turns, slots, n));
        CHECK(got.time * 0.995 <= least * (1.0 + 1e-12));
    }
    // a call's plan below a microsecond, heads of a frame or of millions of tokens in one run
    const auto t0 = std::chrono::steady_clock::now();
    int64_t sum = 0;
    for (int round = 0; round < 200000; ++round) sum += norm_pieces(1, 71145 + 100 * (round % 9000), 3072).pieces;
    const double us = std::chrono::duration<double, std::micro>(std::chrono::steady_clock::now() - t0).count() / 200000;
    if (!(us < 10.0) || sum == 0) { std::printf("%.1f us a plan\n", us); return 1; }
    std::printf("ok\n");
    return 0;
}
