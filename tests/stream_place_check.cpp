// Run on a host by test_stream_places_cpu.py: the places of ragged batches as the kernels compute them.
#include "../paper_2604_20470_amd/csrc/stream_place.h"

#include <cstdio>
#include <cstdlib>
#include <set>
#include <tuple>
#include <vector>

using namespace dr;
using namespace dr::stream;

static uint32_t state = 12345;
static int pick(int lo, int hi) { state = state * 1664525u + 1013904223u; return lo + (int)((state >> 8) % (uint32_t)(hi - lo + 1)); }
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (round %d)\n", __LINE__, #x, round); return 1; } } while (0)

static Place find(const BatchArgs& b, int item, int mul, int tile, int slack) {
    return place_of(b, item, mul, tile, slack, [&](int lo, int step, int hi) {
        int n = 0;
        for (int lane = 0; lane < 64; ++lane) {
            const int64_t i = lo + (int64_t)lane * step;
            n += i < hi && batch_first(b, i < hi ? (int)i : 0, mul, tile, slack) <= item;
        }
        return n;
    });
}

// The lanes of a wave, one to a sequence.
struct Spans {
    std::vector<Span> of;
    template <class F> int total(F&& f) const { int n = 0; for (const Span& s : of) n += f(s); return n; }
    template <class F> int pick(F&& f, int k, int* before) const {
        int n = 0;
        for (size_t s = 0; s < of.size(); ++s) {
            const int x = f(of[s]);
            if (k < n + x) { *before = n; return (int)s; }
            n += x;
        }
        return -1;
    }
    Span at(int s) const { return of.at(s); }
};

int main() {
    for (int round = 0; round < 70000; ++round) {
        // every group of up to 300 heads, some larger ones
        const int group = round < 300 ? round + 1 : pick(1, 65535), r0 = round < 300 ? pick(0, 3) * 256 : pick(0, 1 << 30);
        const Rows256 t = rows_of(r0, group);
        for (int x = 0; x < 256; x += round < 300 ? 1 : 17) {
            int token = -1, head = -1;
            row_at(t, x, &token, &head);
            CHECK(token == (r0 + x) / group && head == (r0 + x) % group);
        }
    }
    for (int round = 0; round < 4000; ++round) {
        const bool garbage = round % 4 == 3;
        const int S = pick(0, 9) ? pick(1, 40) : pick(60, 700), P = 32 << pick(0, 2), pages = pick(1, 50), group = pick(1, 9), R = 16 << pick(0, 4);
        std::vector<int32_t> cu(S + 1), lens(S);
        cu[0] = pick(0, 3) ? 0 : pick(0, 5);
        for (int s = 0; s < S; ++s) {
            const int n = pick(0, 2) ? pick(0, 3) : pick(0, 4 * P);
            cu[s + 1] = cu[s] + n;
            lens[s] = pick(0, 5) ? n + pick(0, 5 * P) : pick(-3, n);
        }
        const int T = pick(0, 3) ? cu[S] : cu[S] + pick(0, 7);
        const int width = pick(0, 12), stride = width + pick(0, 3);
        std::vector<int32_t> table((size_t)S * stride + 1);
        for (auto& p : table) p = pick(0, 6) ? pick(0, pages - 1) : pick(-2, pages + 2);
        if (garbage) {
            const int32_t odd[] = {-2147483647 - 1, -1, 0, 1, 63, 1 << 20, 2147483647};
            for (auto& c : cu) if (!pick(0, 2)) c = odd[pick(0, 6)];
            for (auto& l : lens) if (!pick(0, 1)) l = odd[pick(0, 6)];
            for (auto& p : table) if (!pick(0, 3)) p = odd[pick(0, 6)];
        }
        const BatchArgs b{S, T, width, cu.data(), lens.data(), table.data(), stride};
        // append: every storable token once, nothing outside
        std::set<std::pair<int, int>> stored;
        for (int item = 0; item < T / P + 2 * S; ++item) {
            const Place w = find(b, item, 1, P, 2);
            CHECK(w.seq >= 0 && w.seq < S && (w.n < 0 || (w.begin >= 0 && w.begin + w.n <= T)));
            const Range g = range_of(b, pages, P, w);
            CHECK(g.m >= 0 && g.m <= P);
            if (!g.m) continue;
            CHECK(g.page >= 0 && g.page < pages && g.slot >= 0 && g.slot + g.m <= P && g.token >= 0 && g.token + g.m <= T && g.place % P == g.slot);
            for (int i = 0; i < g.m; ++i) CHECK(stored.insert({w.seq, g.token + i}).second);
        }
        if (!garbage) {
            size_t want = 0;
            for (int s = 0; s < S; ++s)
                for (int t = cu[s]; t < cu[s + 1]; ++t) {
                    const int place = lens[s] - (cu[s + 1] - t);
                    const bool ok = place >= 0 && place / P < width && table[(size_t)s * stride + place / P] >= 0 && table[(size_t)s * stride + place / P] < pages;
                    CHECK(stored.count({s, t}) == (ok ? 1u : 0u));
                    want += ok;
                }
            CHECK(stored.size() == want);
        }
        // attention: every row once, pieces that cover what it sees
        const int splits = pick(1, 64), least = pick(1, 8);
        std::set<std::pair<int, int>> rows;
        for (int64_t item = 0; item < (int64_t)T * group / R + S; ++item) {
            const Place p = find(b, (int)item, group, R, 1);
            Walk w{};
            const bool causal = pick(0, 1);
            if (!walk_of(b, P, R, 64, splits, least, causal, group, p, &w)) continue;
            CHECK(w.begin >= 0 && w.r0 >= 0 && w.r0 < w.rows && w.begin + (w.rows - 1) / group < T);
            CHECK(w.keys >= 0 && w.keys <= width * P && w.active <= splits && w.active >= 0 && (int64_t)w.active * w.per >= w.chunks);
            CHECK((w.active - 1) * (int64_t)w.per < w.chunks || w.chunks == 0);
            for (int r = w.r0; r < w.r0 + R && r < w.rows; ++r) {
                const int n = seen_by(w, causal, group, r);
                CHECK(n >= 0 && n <= w.keys && n <= w.chunks * 64);
                CHECK(rows.insert({w.seq, r}).second);
            }
        }
        if (!garbage) {
            size_t want = 0;
            for (int s = 0; s < S; ++s) want += (size_t)(cu[s + 1] - cu[s]) * group;
            CHECK(rows.size() == want);
        }
        // the same tiles in the order of their keys
        if (S <= 64) {
            const bool causal = pick(0, 1);
            Spans lanes;
            for (int s = 0; s < S; ++s) lanes.of.push_back(span_of(b, P, R, group, s));
            std::set<std::pair<int, int>> tiles;
            int last = 2147483647;
            for (int64_t j = 0; j < (int64_t)T * group / R + S; ++j) {
                const Place p = sorted_place(lanes, R, 64, causal, group, (width * P + 63) / 64, (int)j);
                Walk w{};
                if (!walk_of(b, P, R, 64, splits, least, causal, group, p, &w)) { CHECK(p.n < 0); continue; }
                CHECK(p.seq >= 0 && p.seq < S && w.begin >= 0 && w.r0 >= 0 && w.r0 < w.rows && w.begin + (w.rows - 1) / group < T);
                CHECK(w.chunks <= last && w.keys <= width * P);
                last = w.chunks;
                CHECK(tiles.insert({w.seq, w.r0}).second);
            }
            if (!garbage) {
                size_t want = 0;
                for (int s = 0; s < S; ++s) want += (size_t)((int64_t)(cu[s + 1] - cu[s]) * group + R - 1) / R;
                CHECK(tiles.size() == want);
            }
        }
    }
    std::printf("ok\n");
    return 0;
}
