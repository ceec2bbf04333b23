// How the backward pass of the norms is cut up: plain arithmetic on the host, once a call.  Internal.
#pragma once

#include <stdint.h>

namespace dr {

// Pieces of a run: the number whose rounds take least time, counted in turns of a unit (rows, several at once in a wave); a unit costs some eight of them by itself (its vectors, its
// first rows, its sums).  A round that is not full costs as much as one that is: 21 runs of 3600 tokens of 5120 channels in 49 pieces each are five rounds of 256 workgroups, in 48 four.
// Pieces have four turns at least, and sixteen rounds are the most; of the numbers that take as many rounds the largest takes least, so it is one comparison a round (a search of all numbers
// took the host up to 0.5 ms a call), and of those that give pieces of one length the smallest is taken.
struct NormPieces {
    int64_t pieces;
    double time;
};
inline NormPieces norm_pieces(int64_t runs, int64_t turns, int64_t slots) {
    const int64_t most = turns / 4 > 1 ? turns / 4 : 1;
    NormPieces best{1, (double)((runs + slots - 1) / slots) * (double)(turns + 8)};
    for (int64_t r = 1; r <= 16; ++r) {
        int64_t n = r * slots / runs;
        if (n > most) n = most;
        if (n <= best.pieces) continue;
        const int64_t length = (turns + n - 1) / n;
        n = (turns + length - 1) / length;
        const double time = (double)((runs * n + slots - 1) / slots) * (double)(length + 8);
        if (time < best.time * 0.995) best = NormPieces{n, time};
    }
    return best;
}

}  // namespace dr
