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

// Reading back: the same for tokens that are wanted, from a place before the sequence on if need be.  page < 0: nothing is stored for these m tokens.
DR_HD Range read_range_of(const BatchArgs& b, int pages, int P, const Place& w) {
    Range g{-1, 0, 0, 0, 0};
    if (w.n <= 0 || w.item < 0) return g;
    const int64_t len = b.lens[w.seq], start = len - w.n;
    const int64_t index = (start >= 0 ? start / P : -((P - 1 - start) / P)) + w.item;         // rounded down
    const int64_t from = most64(index * P, start), to = least64((index + 1) * P, len);
    if (from >= to) return g;
    g.page = index >= 0 && index < b.max_pages ? page_of(b, pages, w.seq, (int)index) : -1;
    g.slot = (int)(from - index * P);
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
// len(): tokens in the cache of sequence p.seq.
template <class Len>
DR_HD bool walk_with(Len&& length, const BatchArgs& b, int P, int R, int chunk, int splits, int least, bool causal, int group, const Place& p, Walk* w) {
    if (p.n <= 0 || p.item < 0) return false;
    w->seq = p.seq;
    w->begin = p.begin;
    w->rows = p.n * group;
    if ((int64_t)p.item * R >= w->rows) return false;
    w->r0 = p.item * R;
    const int len = length();
    w->shift = (int64_t)len - p.n;
    w->keys = (int)least64(most64(len, 0), (int64_t)b.max_pages * P);
    w->chunks = (seen_by(*w, causal, group, (int)least64((int64_t)w->r0 + R, w->rows) - 1) + chunk - 1) / chunk;
    w->per = (int)most64((w->chunks + splits - 1) / splits, least);
    w->active = (w->chunks + w->per - 1) / w->per;
    return true;
}

DR_HD bool walk_of(const BatchArgs& b, int P, int R, int chunk, int splits, int least, bool causal, int group, const Place& p, Walk* w) {
    return walk_with([&] { return (int)b.lens[p.seq]; }, b, P, R, chunk, splits, least, causal, group, p, w);
}

// Where the partial sums of a row, head hd of the group of token t.item of its sequence, lie: `pieces` of them, 2^shift (the rows of a tile) slots apart, from slot `first` on. There is
// room for `room` pieces of a tile.  Tiles are head after head, `items` each, those of 256 rows from the last on.
struct Pieces { int64_t first; int pieces; };
// walk(tile): pieces that the tile has.
template <class Walks>
DR_HD Pieces pieces_of(const BatchArgs& b, int shift, int room, int group, int items, bool last_first, const Place& t, int head, int hd, Walks&& walk) {
    const int row = t.item * group + hd, tile = row >> shift;
    const int item = (int)(((int64_t)batch_cu(b, t.seq) * group) >> shift) + t.seq + tile;        // (as batch_first)
    const int64_t at = (int64_t)head * items + (last_first ? items - 1 - item : item);
    return Pieces{(at * room << shift) + (row & ((1 << shift) - 1)), walk(Place{t.seq, t.begin, t.n, tile})};
}

// A window: the token at place i, of frame f = i / frame, sees the keys of frames f - window + 1 .. f and of the first `sinks` ones (below f + 1 too).
struct Window { int32_t frame, window, sinks; };
struct Reach { int lo, hi; };                                 // what a row sees beside the sinks
DR_HD Reach reach_at(const Window& v, int keys, int64_t place) {
    if (place < 0) return Reach{0, 0};
    const int64_t f = (int)place / v.frame;                   // (places fit 32 bits)
    const int hi = (int)least64(keys, (f + 1) * v.frame);
    return Reach{(int)least64(most64((f + 1 - v.window) * v.frame, 0), hi), hi};
}
DR_HD int sink_end(const Window& v, int keys) { return (int)least64((int64_t)v.sinks * v.frame, keys); }
DR_HD bool in_reach(const Reach& r, int sinks, int token) { return (token < r.hi) & ((token >= r.lo) | (token < sinks)); }

// The chunks of keys that a tile's rows see, as one list: those that every row sees whole come first (of the sinks, then of the window), then the edges (of
// the sinks, the window's begin, its end).
struct Chunks { int full0, full1, at1, edge0, at2, edge1, at3, total, sink, low, high; };      // seen: below sink, and low .. high - 1
DR_HD int full_chunks(const Chunks& l) { return l.full0 + l.full1; }
DR_HD int chunk_of(const Chunks& l, int i) {
    int c = i < l.full0 ? i : i - l.full0 + l.at1;
    const int e = i - l.full0 - l.full1;
    c = e >= 0 ? l.full0 + e : c;
    c = e >= l.edge0 ? l.at2 + e - l.edge0 : c;
    return e >= l.edge0 + l.edge1 ? l.at3 + e - l.edge0 - l.edge1 : c;
}
DR_HD Chunks window_chunks(const Window& v, int keys, int64_t first, int64_t last, int chunk) {      // places of the first row and the last
    const Reach a = reach_at(v, keys, first), z = reach_at(v, keys, last);
    int sink = sink_end(v, keys), lo0 = a.lo, lo1 = z.lo;     // (all of them grow from row to row)
    if (lo1 <= (sink < a.hi ? sink : a.hi)) lo0 = lo1 = sink = 0;        // no row has anything between its sinks and its window
    const int s0 = sink < a.hi ? sink : a.hi, s1 = sink < z.hi ? sink : z.hi;
    Chunks l;
    l.full0 = s0 / chunk;
    const int sinks = (s1 + chunk - 1) / chunk, end = (z.hi + chunk - 1) / chunk;
    l.at2 = lo0 / chunk > sinks ? lo0 / chunk : sinks;        // the window's first chunk
    if (l.at2 > end) l.at2 = end;
    const int w0 = (lo1 + chunk - 1) / chunk, w1 = a.hi / chunk;
    l.at1 = w0 < l.at2 ? l.at2 : w0 > end ? end : w0;
    l.at3 = w1 < l.at1 ? l.at1 : w1 > end ? end : w1;
    l.full1 = l.at3 - l.at1;
    l.edge0 = sinks - l.full0;
    l.edge1 = l.at1 - l.at2;
    l.total = sinks + end - l.at2;
    l.sink = s1;
    l.low = lo0;
    l.high = z.hi;
    return l;
}
// Whether some row sees one of the `n` tokens from `place` on.
DR_HD bool any_seen(const Chunks& l, int64_t place, int n) { return (place < l.sink) | ((place + n > l.low) & (place < l.high) & (l.low < l.high)); }
template <class Len>
DR_HD bool window_walk_with(Len&& length, const BatchArgs& b, int P, int R, int chunk, int splits, int least, const Window& v, int group, const Place& p, Walk* w, Chunks* l) {
    if (!walk_with(length, b, P, R, chunk, splits, least, false, group, p, w)) return false;
    const int last = (int)least64((int64_t)w->r0 + R, w->rows) - 1;
    *l = window_chunks(v, w->keys, w->shift + w->r0 / group, w->shift + last / group, chunk);
    w->chunks = l->total;
    w->per = (int)most64((w->chunks + splits - 1) / splits, least);
    w->active = (w->chunks + w->per - 1) / w->per;
    return true;
}
// Chunks that a tile of a sequence of n new tokens and `len` in all has at most; window.frame = 0: there is no window.
DR_HD int most_chunks(const BatchArgs& b, int P, int chunk, const Window& v, int n, int len, int group, int shift) {
    const int64_t keys = least64(most64(len, 0), (int64_t)b.max_pages * P), all = (keys + chunk - 1) / chunk;
    if (v.frame == 0) return (int)all;
    const int64_t tokens = least64(n, (1 << shift) / group + 2);              // of a tile, or one more
    return (int)least64(all, (((int64_t)v.window + v.sinks) * v.frame + tokens + v.frame) / chunk + 4);
}
DR_HD bool window_walk_of(const BatchArgs& b, int P, int R, int chunk, int splits, int least, const Window& v, int group, const Place& p, Walk* w, Chunks* l) {
    return window_walk_with([&] { return (int)b.lens[p.seq]; }, b, P, R, chunk, splits, least, v, group, p, w, l);
}

// How the pieces of keys are cut, where the device decides it.  The kernel that writes partial sums and the one that joins them each work it out: whole numbers
// only, so that both come to the same however they are compiled (a sum of products in fp32, contracted in one of them, differs from 2^24 chunks on).
// Chunks of a piece of the rows kernel: `all` chunks (below 2^50) in `budget` pieces, but no more than `splits` pieces of the longest tile, `least` at least, whole turns of the waves.
// (Divisions of 32 bits, coarser from 2^31 chunks on: in 64 bits they cost a call 0.5 us.)
DR_HD int piece_chunks(int64_t all, int budget, int longest, int splits, int least, int waves) {
    int coarse = 0;
    while ((all >> coarse) >= (1ll << 31)) ++coarse;
    const uint32_t share = ((uint32_t)(all >> coarse) + (uint32_t)budget - 1) / (uint32_t)budget;
    const int even = (int)least64((int64_t)share << coarse, 1000000000), room = (longest + splits - 1) / splits;
    const int size = even > room ? even : room;
    return ((size > least ? size : least) + waves - 1) / waves * waves;
}
// What pieces of `size` chunks take, `slots` of them at once, a piece costing some three chunks by itself; and whether that is less than `best` by more than 3 %.
DR_HD int64_t pieces_cost(int pieces, int slots, int size) { return (int64_t)((pieces + slots - 1) / slots) * (size + 3); }
DR_HD bool cheaper(int64_t cost, int64_t best) { return cost * 100 < best * 97; }
// A number of chunks that may be large as two that 64 lanes can add up in 32 bits (tiles below 2^24 in all, chunks of one up to 2^25).
DR_HD int low_part(int64_t chunks) { return (int)(chunks & 0xffffff); }
DR_HD int high_part(int64_t chunks) { return (int)(chunks >> 24); }
DR_HD int64_t from_parts(int low, int high) { return ((int64_t)high << 24) + low; }
// What a tile's keys take in the many-rows kernel, `rest` tiles in `pieces` each (64 at most) and `chip` of them at once, a piece costing `piece` chunks by itself: in 64ths of a chunk, coarser
// from 2^17 chunks on.  And whether a cost is within 1 % of the least.
DR_HD int tiles_cost(int longest, int pieces, int rest, int chip, int piece) {
    int coarse = 0;
    while (coarse < 14 && (longest >> coarse) >= (1 << 17)) ++coarse;
    return (rest * pieces + chip - 1) / chip * ((int)(((int64_t)longest << 6) >> coarse) / pieces + ((piece << 6) >> coarse));
}
DR_HD bool near_least(int cost, int least) { return (int64_t)cost * 99 <= (int64_t)least * 100; }

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
