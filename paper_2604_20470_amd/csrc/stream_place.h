// Which work item of a ragged batch is what: plain integer arithmetic, the same on the device and on a host.  Every access of
// the append and of the cached attention follows from these numbers, whatever the batch's arrays hold.  Internal.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define DR_HD __host__ __device__ __forceinline__
#else
#define DR_HD inline
#endif

namespace dr {

struct BatchArgs {
    int32_t sequences, tokens, max_pages;
    const int32_t *cu, *lens, *page_table;
    int64_t table_stride;
};

namespace stream {

DR_HD int64_t least64(int64_t a, int64_t b) { return a < b ? a : b; }
DR_HD int64_t most64(int64_t a, int64_t b) { return a > b ? a : b; }

// Places of a ragged batch: sequence s owns the work items first(s) .. first(s + 1) - 1, first(s) = floor(cu[s] * mul / tile) + slack * s.
// Since floor(x + y) >= floor(x) + floor(y), that leaves a sequence of n tokens at least floor(n * mul / tile) + slack items, without
// sums over the sequences before it and with a number of items, floor(tokens * mul / tile) + slack * sequences, that the host knows.
struct Place { int seq, begin, n, item; };                                    // n < 0: no sequence

DR_HD int batch_cu(const BatchArgs& b, int s) { return (int)least64(most64(b.cu[s], 0), b.tokens); }
DR_HD int batch_first(const BatchArgs& b, int s, int mul, int tile, int slack) { return (int)((int64_t)batch_cu(b, s) * mul / tile) + slack * s; }

// The last sequence that begins at or before the item.  count(lo, step, hi): how many of lo, lo + step, ... (64 at most, below hi) do.
template <class Count>
DR_HD Place place_of(const BatchArgs& b, int item, int mul, int tile, int slack, Count&& count) {
    int lo = 0, hi = b.sequences;
    Place p{0, 0, -1, 0};
    while (hi > lo) {
        const int step = (hi - lo + 63) / 64, n = count(lo, step, hi);
        if (n == 0) return p;                                                 // (in the first turn only: items before the first sequence)
        lo += (n - 1) * step;
        if (step == 1) break;
        hi = (int)least64(hi, lo + step);
    }
    p.seq = lo;
    p.begin = batch_cu(b, lo);
    p.n = (int)most64(batch_cu(b, lo + 1) - p.begin, 0);
    p.item = item - batch_first(b, lo, mul, tile, slack);
    return p;
}

// A page of the pool, or -1 (outside the table or the pool).
DR_HD int page_of(const BatchArgs& b, int pages, int seq, int index) {
    if (index < 0 || index >= b.max_pages) return -1;
    const int p = b.page_table[(int64_t)seq * b.table_stride + index];
    return p >= 0 && p < pages ? p : -1;
}

// Append: the new tokens of one page, slots slot .. slot + m - 1, from row `token` on; m = 0: nothing to do.
struct Range { int page, slot, m, token, place; };
DR_HD Range range_of(const BatchArgs& b, int pages, int P, const Place& w) {
    Range g{-1, 0, 0, 0, 0};
    if (w.n <= 0) return g;
    const int len = b.lens[w.seq];
    const int64_t start = (int64_t)len - w.n;                 // place of the first new token; negative: that many are not stored
    const int64_t first = most64(start, 0), index = first / P + w.item;
    const int64_t from = most64(index * P, first), to = least64((index + 1) * P, len);
    if (w.item < 0 || from >= to || index >= b.max_pages) return g;
    g.page = page_of(b, pages, w.seq, (int)index);
    if (g.page < 0) return g;
    g.slot = (int)(from % P);
    g.m = (int)(to - from);
    g.place = (int)from;
    g.token = w.begin + (int)(from - start);
    return g;
}

// Attention: what a tile of R rows, (token, head of the group) pairs, has to walk.
struct Walk {
    int seq, begin, r0, rows, keys;                           // rows of the sequence; keys: places that the table holds
    int64_t shift;                                            // place of the first new token
    int chunks, per, active;                                  // chunks of keys in all, of a piece; pieces that have any
};
DR_HD int seen_at(const Walk& w, bool causal, int token) { return causal ? (int)least64(w.keys, most64(w.shift + token + 1, 0)) : w.keys; }
DR_HD int seen_by(const Walk& w, bool causal, int group, int row) { return seen_at(w, causal, row / group); }

// Token of the sequence, and head of the group, of a row by its place (0 .. 255) in the tile.  A division costs some forty instructions; this
// multiplies with 2^20 / group, which is exact for the 511 and less that it is taken of.  Groups above 256: a tile has two tokens at most.
struct Rows256 { int token, head, group, inverse; };
DR_HD Rows256 rows_of(int r0, int group) { return Rows256{r0 / group, r0 % group, group, (1 << 20) / group + 1}; }
DR_HD void row_at(const Rows256& t, int place, int* token, int* head) {
    const int x = t.head + place, q = t.group > 256 ? (x >= t.group ? 1 : 0) : (x * t.inverse) >> 20;
    *token = t.token + q;
    *head = x - q * t.group;
}
DR_HD bool walk_of(const BatchArgs& b, int P, int R, int chunk, int splits, int least, bool causal, int group, const Place& p, Walk* w) {
    if (p.n <= 0 || p.item < 0) return false;
    w->seq = p.seq;
    w->begin = p.begin;
    w->rows = p.n * group;
    if ((int64_t)p.item * R >= w->rows) return false;
    w->r0 = p.item * R;
    const int len = b.lens[p.seq];
    w->shift = (int64_t)len - p.n;
    w->keys = (int)least64(most64(len, 0), (int64_t)b.max_pages * P);
    w->chunks = (seen_by(*w, causal, group, (int)least64((int64_t)w->r0 + R, w->rows) - 1) + chunk - 1) / chunk;
    w->per = (int)most64((w->chunks + splits - 1) / splits, least);
    w->active = (w->chunks + w->per - 1) / w->per;
    return true;
}

// Tiles in the order of their keys, most first: a batch of unequal sequences then ends with its shortest tiles on all compute units.
struct Span { int begin, n, rows, tiles, keys; int64_t shift; };
DR_HD Span span_of(const BatchArgs& b, int P, int R, int group, int seq) {
    Span s{};
    s.begin = batch_cu(b, seq);
    s.n = (int)most64(batch_cu(b, seq + 1) - s.begin, 0);
    s.rows = s.n * group;
    s.tiles = (int)(((int64_t)s.rows + R - 1) / R);
    s.keys = (int)least64(most64(b.lens[seq], 0), (int64_t)b.max_pages * P);
    s.shift = (int64_t)b.lens[seq] - s.n;
    return s;
}
// How many tiles of a sequence have c chunks of keys at least: its last ones.
DR_HD int tiles_with(const Span& s, int R, int chunk, bool causal, int group, int c) {
    if (c <= 0) return s.tiles;
    const int64_t before = (int64_t)(c - 1) * chunk;                          // its last row has to see the key behind these
    if (s.keys <= before) return 0;
    if (!causal) return s.tiles;
    const int64_t row = (before - s.shift) * group;                           // the first row that does
    return row <= 0 ? s.tiles : row >= s.rows ? 0 : s.tiles - (int)(row / R);
}
// Tile j of that order.  `lanes` has the spans: total(f) sums f over them, pick(f, k, &before) finds the one that holds the k-th of all f's.
template <class Lanes>
DR_HD Place sorted_place(Lanes& lanes, int R, int chunk, bool causal, int group, int chunks, int j) {
    auto with = [&](int c) { return [=](const Span& s) { return tiles_with(s, R, chunk, causal, group, c); }; };
    Place p{0, 0, -1, 0};
    if (j >= lanes.total(with(0))) return p;
    int lo = 0, hi = chunks + 1, more = 0;                                    // total(lo) > j >= total(hi) = more
    while (hi - lo > 1) {
        const int c = lo + (hi - lo) / 2, n = lanes.total(with(c));
        if (n > j) lo = c;
        else { hi = c; more = n; }
    }
    int before = 0;
    p.seq = lanes.pick([&](const Span& s) { return tiles_with(s, R, chunk, causal, group, lo) - tiles_with(s, R, chunk, causal, group, hi); }, j - more, &before);
    const Span s = lanes.at(p.seq);
    p.begin = s.begin;
    p.n = s.n;
    p.item = s.tiles - tiles_with(s, R, chunk, causal, group, lo) + (j - more - before);
    return p;
}

// Rotation: unit u of a head is W pairs, u W .. u W + W - 1, or 2 W channels behind `dim` that are copied (dim is a multiple of 2 W here).  Pairs below end0
// go by axis 0, below end1 by axis 1.  A unit that is copied has no axis, so nothing is read for it: behind the last pair there may be no third
// row of positions, or no second.
DR_HD int pair_axis(int end0, int end1, int pair) { return (pair >= end0) + (pair >= end1); }
// The positions of unit u's pairs: read(axis) is called once for each axis in turn, use(j, pair, position) for every pair.
template <int W, class Read, class Use>
DR_HD bool unit_positions(int dim, int end0, int end1, int u, Read&& read, Use&& use) {
    if (2 * W * u >= dim) return false;
    int axis = -1, pos = 0;
#ifdef __HIPCC__
#pragma unroll
#endif
    for (int j = 0; j < W; ++j) {
        const int pair = u * W + j, k = pair_axis(end0, end1, pair);
        if (k != axis) pos = read(k);
        axis = k;
        use(j, pair, pos);
    }
    return true;
}

// Tokens of one launch of the rotation, of N with `units` threads each: a launch holds fewer than 2^32 threads along one axis.
DR_HD int rope_tokens_of_a_launch(int N, int units, int threads) {
    const int64_t most = ((1ll << 32) / threads - 1) * threads / units;
    return (int)least64(N, most);
}

}  // namespace stream
}  // namespace dr
