// Run on a host by test_stream_views_cpu.py: places of tokens that are read back, the chunks of windows, the slots of partial sums.
#include "../paper_2604_20470_amd/csrc/stream_place.h"

#include <cstdio>
#include <cstdlib>
#include <map>
#include <set>
#include <vector>

using namespace dr;
using namespace dr::stream;

static uint32_t state = 4321;
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
static bool sees(const Window& v, int keys, int64_t place, int j) {
    if (place < 0 || j >= keys) return false;
    const int64_t f = place / v.frame, g = j / v.frame;
    return g <= f && (f - g < v.window || g < v.sinks);
}

int main() {
    // a window's list of chunks: all that some row sees, nothing twice, the first part seen whole by every row
    for (int round = 0; round < 6000; ++round) {
        const Window v{pick(0, 2) ? 1 : pick(1, 300), pick(0, 1) ? pick(1, 12) : pick(1, 700), pick(0, 1) ? 0 : pick(1, 150)};
        const int keys = pick(0, 1500), span = pick(0, 260);
        const int64_t first = pick(-40, 1500), last = first + span;
        const Chunks l = window_chunks(v, keys, first, last, 64);
        CHECK(l.full0 >= 0 && l.full1 >= 0 && l.edge0 >= 0 && l.edge1 >= 0 && l.total >= full_chunks(l) + l.edge0 + l.edge1);
        std::set<int> have;
        for (int i = 0; i < l.total; ++i) {
            const int c = chunk_of(l, i);
            CHECK(c >= 0 && c * 64 < keys + 63);
            CHECK(have.insert(c).second);
            if (i >= full_chunks(l)) continue;
            for (int64_t p = first; p <= last; p += last > first ? last - first : 1)
                for (int j = 64 * c; j < 64 * c + 64; ++j) CHECK(sees(v, keys, p, j));
            const int64_t mid = first + pick(0, span);
            for (int j = 64 * c; j < 64 * c + 64; ++j) CHECK(sees(v, keys, mid, j));
        }
        std::set<int> want;
        for (int64_t p = first; p <= last; ++p) {
            const Reach r = reach_at(v, keys, p);
            const int sink = sink_end(v, keys);
            for (int j = 0; j < keys; ++j) {
                const bool s = sees(v, keys, p, j);
                CHECK(in_reach(r, sink, j) == s);
                if (s) want.insert(j / 64);
            }
            if (span > 40) p += 3;
        }
        for (int c : want) CHECK(have.count(c));
        for (int j = 0; j < keys; j += 32) {                // half chunks that some row sees
            bool any = false;
            for (int64_t p = first; p <= last; ++p)
                for (int i = j; i < j + 32; ++i) any = any || sees(v, keys, p, i);
            CHECK(any_seen(l, j, 32) == any || (!have.count(j / 64) && !any));
        }
        {
            const int32_t cu[2] = {0, span + 1}, len[1] = {(int32_t)(last + 1)};
            const BatchArgs one{1, span + 1, (keys + 31) / 32, cu, len, nullptr, 64};
            CHECK(l.total <= most_chunks(one, 32, 64, v, span + 1, (int)(last + 1), 1, 8) || last + 1 < keys || span > 256);
        }
        // (at most the ends' chunks beyond what is seen: a tile never walks what lies between sinks and window)
        CHECK(l.total <= (int)want.size() + 2);
    }
    {
        const int round = -1;
        const int most = 1 << 30;
        const Window v{most, most, most}, u{most, 1, 0}, t{1, most, most};
        CHECK(reach_at(v, most - 1, 2147483646).hi == most - 1 && reach_at(v, most - 1, 2147483646).lo == 0 && sink_end(v, most - 1) == most - 1);
        CHECK(reach_at(u, most - 1, 5).lo == 0 && reach_at(u, most - 1, 5).hi == most - 1 && reach_at(u, 100, 2147483646).lo == 100);
        CHECK(reach_at(t, most - 1, 77).hi == 78 && reach_at(t, most - 1, 77).lo == 0);
    }
    for (int round = 0; round < 3000; ++round) {
        const bool garbage = round % 4 == 3;
        const int S = pick(0, 9) ? pick(1, 40) : pick(60, 400), P = 32 << pick(0, 2), pages = pick(1, 50), group = pick(1, 9), heads = pick(1, 5);
        std::vector<int32_t> cu(S + 1), lens(S);
        cu[0] = pick(0, 3) ? 0 : pick(0, 5);
        for (int s = 0; s < S; ++s) {
            const int n = pick(0, 2) ? pick(0, 3) : pick(0, 4 * P);
            cu[s + 1] = cu[s] + n;
            lens[s] = pick(0, 5) ? n + pick(0, 5 * P) : pick(-300, n);
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
        // read: every token of a sequence once
        std::map<std::pair<int, int>, int> page;
        for (int item = 0; item < T / P + 2 * S; ++item) {
            const Range g = read_range_of(b, pages, P, find(b, item, 1, P, 2));
            CHECK(g.m >= 0 && g.m <= P);
            if (!g.m) continue;
            const int seq = find(b, item, 1, P, 2).seq;
            CHECK(g.page >= -1 && g.page < pages && g.slot >= 0 && g.slot + g.m <= P && g.token >= 0 && g.token + g.m <= T);
            for (int i = 0; i < g.m; ++i) CHECK(page.insert({{seq, g.token + i}, g.page < 0 ? -1 : g.page * P + g.slot + i}).second);
        }
        if (!garbage) {
            size_t want = 0;
            for (int s = 0; s < S; ++s)
                for (int t = cu[s]; t < cu[s + 1]; ++t, ++want) {
                    const int place = lens[s] - (cu[s + 1] - t), index = place >= 0 ? place / P : -1;
                    const int p = index >= 0 && index < width ? table[(size_t)s * stride + index] : -1;
                    CHECK(page.count({s, t}) && (page[{s, t}]) == (p >= 0 && p < pages ? p * P + place % P : -1));
                }
            CHECK(page.size() == want);
        }
        // slots of partial sums: what the tile of a row writes is what the row's token finds, and all of it lies in the scratch
        const int splits = pick(1, 64), least = pick(1, 8), shift = pick(0, 1) ? 8 : pick(4, 5), R = 1 << shift;
        const bool causal = pick(0, 1), last_first = R == 256;
        const int items = (int)((int64_t)T * group / R + S);
        std::map<std::pair<int, int>, std::pair<int64_t, int>> wrote;
        for (int at = 0; at < items; ++at) {
            Walk w{};
            const Place q = find(b, last_first ? items - 1 - at : at, group, R, 1);
            if (!walk_of(b, P, R, 64, splits, least, causal, group, q, &w)) continue;
            CHECK(w.chunks <= most_chunks(b, P, 64, Window{0, 0, 0}, q.n, lens[q.seq], group, shift));
            for (int r = w.r0; r < w.r0 + R && r < w.rows; ++r) wrote[{w.seq, r}] = {(int64_t)at * splits * R + r - w.r0, w.active};
        }
        for (int t = 0; t < T; t += garbage ? 3 : 1) {
            const Place p = find(b, t, 1, 1, 0);
            if (p.n <= 0 || p.item < 0 || p.item >= p.n) {
                if (!garbage) CHECK(t < cu[0] || t >= cu[S]);
                continue;
            }
            const int head = pick(0, heads - 1), hd = pick(0, group - 1);
            const Pieces x = pieces_of(b, shift, splits, group, items, last_first, p, head, hd, [&](const Place& q) { Walk w; return walk_of(b, P, R, 64, splits, least, causal, group, q, &w) ? w.active : 0; });
            CHECK(x.pieces >= 0 && x.pieces <= splits && x.first >= 0);
            CHECK(x.pieces == 0 || x.first + (int64_t)(x.pieces - 1) * R < (int64_t)items * heads * splits * R);
            if (garbage) continue;
            CHECK(t == cu[p.seq] + p.item && wrote.count({p.seq, p.item * group + hd}));
            const auto y = wrote[{p.seq, p.item * group + hd}];
            CHECK(x.pieces == y.second && x.first == y.first + (int64_t)head * items * splits * R);
        }
        // windows over garbage too: chunks of a tile lie in the table, pieces cover them
        const Window v{pick(0, 1) ? 1 : pick(1, 1 << 30), pick(0, 1) ? pick(1, 300) : pick(1, 1 << 30), pick(0, 1) ? pick(0, 200) : pick(0, 1 << 30)};
        for (int at = 0; at < items; ++at) {
            Walk w{};
            Chunks l{};
            const Place p = find(b, at, group, R, 1);
            if (!window_walk_of(b, P, R, 64, splits, least, v, group, p, &w, &l)) continue;
            CHECK(l.total <= most_chunks(b, P, 64, v, p.n, lens[p.seq], group, shift));
            CHECK(w.chunks == l.total && w.chunks >= 0 && w.active <= splits && (int64_t)w.active * w.per >= w.chunks && ((w.active - 1) * (int64_t)w.per < w.chunks || w.chunks == 0));
            for (int i = 0; i < w.chunks; ++i) CHECK(chunk_of(l, i) >= 0 && (int64_t)chunk_of(l, i) * 64 < (int64_t)width * P);
        }
    }
    std::printf("ok\n");
    return 0;
}
