// Run on a host by test_stream_pairs_cpu.py: which positions a rotation reads for a unit of pairs, in an array that has the entries it needs and no
// others (the sanitizers see any access beside it).
#include "../paper_2604_20470_amd/csrc/stream_place.h"

#include <cstdio>
#include <vector>

using namespace dr::stream;

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (d %d dim %d axes %d unit %d)\n", __LINE__, #x, d, dim, axes, u); return 1; } } while (0)

template <int W>
static int check() {
    const int tokens = 5;
    for (int d = 64; d <= 256; d += 64)
        for (int dim = 0; dim <= d; dim += 2 * W)
            for (int axes = 1; axes <= 3; ++axes)
                for (int cut = 0; cut <= dim / 2; cut += axes == 1 ? dim / 2 + 1 : 1) {
                    // pairs of each axis; some have none
                    int n[3] = {axes == 1 ? dim / 2 : cut, 0, 0};
                    if (axes == 2) n[1] = dim / 2 - cut;
                    if (axes == 3) { n[1] = (dim / 2 - cut) / 3; n[2] = dim / 2 - cut - n[1]; }
                    const std::vector<int> positions((size_t)axes * tokens, 7);
                    for (int u = 0; u < d / (2 * W); ++u)
                        for (int token = 0; token < tokens; ++token) {
                            int used = 0;
                            const bool turned = unit_positions<W>(dim, n[0], n[0] + n[1], u, [&](int axis) { return positions.at((size_t)axis * tokens + token); },
                                                                  [&](int j, int pair, int pos) {
                                                                      int axis = 0, upto = n[0];
                                                                      while (pair >= upto) upto += n[++axis];
                                                                      used += j == used && pair == u * W + j && pair < dim / 2 && pos == 7 && axis < axes;
                                                                  });
                            CHECK(turned == (2 * W * u < dim) && used == (turned ? W : 0));
                        }
                }
    return 0;
}

int main() {
    if (check<4>() || check<8>()) return 1;
    std::printf("ok\n");
    return 0;
}
