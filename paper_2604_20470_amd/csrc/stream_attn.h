// What the kernels of the attention over the paged cache share.  Internal: not part of the public ABI.
#pragma once

#include "stream_common.h"

#include <type_traits>

namespace dr {
namespace stream {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4, kChunk = 64;
constexpr float kLn2 = 0.69314718055994530942f;
// What a piece of a tile in a window costs by itself, in chunks: its first chunk, its partial sums, the join.  Behind tiles that stay whole it gains less, since those do not end together
// (8 ragged prompts, 24 heads on 8, a window of 1024, the last 80 of 1104 tiles in pieces: 281 us, whole 253; 256 tokens of 40 heads, the same window, 40 tiles in pieces: 71, whole 91).
DR_HD int window_piece(bool all) { return all ? 8 : 16; }
// Tiles of a round of the many-rows kernel, which has one workgroup on a compute unit: a multiple of the eight XCDs.
DR_HD int tile_round(int cus) { return (int)most64(cus / 8 * 8, 8); }

// What the kernels are built for: all of the cache, a window of it, or all of it with partial sums as the results whatever the number of pieces.
enum Mode { kAll = 0, kWindow = 1, kParts = 2 };

struct Args {
    CacheArgs c;
    BatchArgs b;
    const char* q;
    char* o;
    int64_t qt, qh, ot, oh;               // bytes
    float* lse;
    float* part_o;                        // [workgroups - whole][splits][rows][D]
    float4* part_sums;                    // [workgroups - whole][splits][rows]: reference, sum, divisor
    int32_t group, causal, splits, least; // query heads to a cached one; pieces at most; chunks of a piece at least
    int32_t workgroups;                   // tiles of rows of all sequences and cached heads
    int32_t whole;                        // tiles below are not cut into pieces
    float scale;                          // log2(e) / sqrt(D)
    Window window;                        // kWindow
    int32_t budget, cus;                  // not kAll: pieces that the rows kernel's workgroups share out, or that the many-rows kernel has room for; compute units
};

// The walk of a work item, in scalars: it is the same in every lane, and control flow that the compiler takes for divergent has
// cost correctness here (moves of live ranges put in front of the join's exec mask, in kernels that use most registers).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <int R>
__device__ __forceinline__ bool walk_to(const Args& a, Place p, int splits, Walk* w) {
    p.seq = uniform(p.seq);
    p.begin = uniform(p.begin);
    p.n = uniform(p.n);
    p.item = uniform(p.item);
    const bool any = walk_of(a.b, a.c.page_tokens, R, kChunk, splits, a.least, a.causal, a.group, p, w);
    if (!uniform(any)) return false;
    w->keys = uniform(w->keys);
    w->shift = ((int64_t)uniform((int)(w->shift >> 32)) << 32) | (uint32_t)uniform((int)w->shift);
    w->chunks = uniform(w->chunks);
    w->per = uniform(w->per);
    w->active = uniform(w->active);
    return true;
}

// The same where the sequence's tokens in the cache are known, and over a window.
__device__ __forceinline__ bool known_walk_to(const Args& a, int R, const Place& p, int len, int splits, int least, Walk* w) {
    const bool any = walk_with([&] { return len; }, a.b, a.c.page_tokens, R, kChunk, splits, least, a.causal, a.group, p, w);
    if (!uniform(any)) return false;
    w->keys = uniform(w->keys);
    w->shift = ((int64_t)uniform((int)(w->shift >> 32)) << 32) | (uint32_t)uniform((int)w->shift);
    w->chunks = uniform(w->chunks);
    w->per = uniform(w->per);
    w->active = uniform(w->active);
    return true;
}
__device__ __forceinline__ bool window_walk_to(const Args& a, int R, const Place& p, int len, int splits, int least, Walk* w, Chunks* l) {
    const bool any = window_walk_with([&] { return len; }, a.b, a.c.page_tokens, R, kChunk, splits, least, a.window, a.group, p, w, l);
    if (!uniform(any)) return false;
    w->keys = uniform(w->keys);
    w->shift = ((int64_t)uniform((int)(w->shift >> 32)) << 32) | (uint32_t)uniform((int)w->shift);
    w->chunks = uniform(w->chunks);
    w->per = uniform(w->per);
    w->active = uniform(w->active);
    l->full0 = uniform(l->full0);
    l->full1 = uniform(l->full1);
    l->at1 = uniform(l->at1);
    l->edge0 = uniform(l->edge0);
    l->at2 = uniform(l->at2);
    l->edge1 = uniform(l->edge1);
    l->at3 = uniform(l->at3);
    l->sink = uniform(l->sink);
    l->low = uniform(l->low);
    l->high = uniform(l->high);
    return true;
}

template <int R>
__device__ __forceinline__ bool tile_walk(const Args& a, int item, int splits, Walk* w) { return walk_to<R>(a, find_place(a.b, item, a.group, R, 1), splits, w); }

__device__ __forceinline__ Rows256 uniform_rows(int r0, int group) {
    const Rows256 t = rows_of(r0, group);
    return Rows256{uniform(t.token), uniform(t.head), group, uniform(t.inverse)};
}

// A lane to a sequence, for whole waves.
struct SpanLanes {
    Span mine;
    __device__ __forceinline__ SpanLanes(const BatchArgs& b, int P, int R, int group) {
        const int s = threadIdx.x & 63;
        mine = span_of(b, P, R, group, min(s, b.sequences - 1));
        if (s >= b.sequences) mine.tiles = mine.rows = mine.keys = 0;
    }
    // sums of the lanes up to this one
    static __device__ __forceinline__ int scan(int x) {
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // within rows of 16: 1, 2, 4, 8 lanes up
        x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // a row's last lane to the next row, the first half's to the second
        x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
        return x;
    }
    template <class F>
    __device__ __forceinline__ int total(F&& f) const { return __builtin_amdgcn_readlane(scan(f(mine)), 63); }
    template <class F>
    __device__ __forceinline__ int pick(F&& f, int k, int* before) const {
        const int x = f(mine), upto = scan(x);
        const int s = min(__popcll(__ballot(upto <= k)), 63);
        *before = __builtin_amdgcn_readlane(upto - x, s);
        return s;
    }
    __device__ __forceinline__ Span at(int s) const {
        Span r;
        r.begin = __builtin_amdgcn_readlane(mine.begin, s);
        r.n = __builtin_amdgcn_readlane(mine.n, s);
        r.rows = __builtin_amdgcn_readlane(mine.rows, s);
        r.tiles = __builtin_amdgcn_readlane(mine.tiles, s);
        r.keys = __builtin_amdgcn_readlane(mine.keys, s);
        r.shift = ((int64_t)__builtin_amdgcn_readlane((int)(mine.shift >> 32), s) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)mine.shift, s);
        return r;
    }
};
// f over all lanes of values >= 0 (0 where a lane has none).
template <class T, class F>
__device__ __forceinline__ T over_lanes(T x, F&& f) {
    auto step = [&](auto ctrl, auto rows) {
        x = f(x, __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false)));
    };
    using std::integral_constant;
    step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
    step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
// Up to 64 sequences, a lane to each (not kAll): its place in the batch, its tiles and the chunks that one of them has at most.
struct SequenceLanes {
    int begin, n, len, first, tiles, chunks;
    __device__ __forceinline__ void read(const Args& a, int shift) {
        const int lane = threadIdx.x & 63, s = min(lane, a.b.sequences - 1), items = a.workgroups / a.c.heads;
        begin = batch_cu(a.b, s);
        n = max(batch_cu(a.b, s + 1) - begin, 0);
        len = a.b.lens[s];
        if (lane >= a.b.sequences) n = 0;
        first = (int)(((int64_t)begin * a.group) >> shift) + s;               // (as batch_first)
        tiles = (int)(((int64_t)n * a.group + (1 << shift) - 1) >> shift);
        // (sequences that overlap would have more than the batch has room for)
        tiles = min(tiles, items + 1);
        if (SpanLanes::scan(tiles) > items) n = tiles = 0;
        chunks = n > 0 ? most_chunks(a.b, a.c.page_tokens, kChunk, a.window, n, len, a.group, shift) : 0;
    }
    __device__ __forceinline__ Place place(int seq, int item, int* length) const {
        *length = __builtin_amdgcn_readlane(len, seq);
        return Place{seq, __builtin_amdgcn_readlane(begin, seq), __builtin_amdgcn_readlane(n, seq), item};
    }
};
// The pieces of the rows kernel (not kAll), for whole waves.  Up to 64 sequences: a lane to a sequence, which has the tiles and chunks that it has, not those of the longest; a piece has as many chunks
// as give `budget` pieces in all.  Beyond: every tile in a.splits pieces at most, as the host has planned.
struct Shares : SequenceLanes {
    int shift, per, total;                      // log2 of a tile's rows; chunks of a piece (0: by a.splits and a.least); pieces
    int upto;                                   // pieces of this lane's sequence and those before
    __device__ __forceinline__ Shares(const Args& a, int log2_rows) : shift(log2_rows), per(0) {
        total = a.workgroups * a.splits;
        if (a.b.sequences > 64) return;
        read(a, shift);
        if (a.splits > 1) {
            const int64_t mine = (int64_t)tiles * a.c.heads * chunks;
            auto sum = [](int x, int y) { return x + y; };
            const int64_t all = from_parts(over_lanes(low_part(mine), sum), __any(high_part(mine) != 0) ? over_lanes(high_part(mine), sum) : 0);
            const int longest = over_lanes(chunks, [](int x, int y) { return max(x, y); });
            // (no more pieces of a tile than the scratch has room for; whole turns of the four waves)
            per = uniform(piece_chunks(all, a.budget, longest, a.splits, a.least, kWaves));
        } else {
            per = 1 << 29;
        }
        auto cut = [&](int size) { return SpanLanes::scan(tiles * a.c.heads * max((chunks + size - 1) / size, 1)); };
        upto = cut(per);
        total = __builtin_amdgcn_readlane(upto, 63);
        // A round of pieces that is not full takes as long as one that is: of this size and the next two the one whose rounds take least, a piece costing some three chunks by itself
        // (8 sequences of 4 tokens, 40 heads on 8, a window of 4096: 576 pieces of 8 chunks on 512 workgroups 50 us, 384 of 12 41; 64 single tokens, a window of 1024: 53 and 46; what it costs is 0.5 us).
        // Beside a prefix as much is lost as won: 40 sequences in two groups 93 and 81, 48 in one 105 and 107, in fp32 115 and 117.
        const int slots = 2 * a.cus;
        if (a.window.frame && a.splits > 1 && total > slots) {
            int64_t best = pieces_cost(total, slots, per);
            for (int i = 1, size = per; i < 3; ++i) {
                size += kWaves;
                const int more = cut(size), pieces = __builtin_amdgcn_readlane(more, 63);
                const int64_t cost = pieces_cost(pieces, slots, size);
                if (cheaper(cost, best)) {
                    best = cost;
                    per = size;
                    upto = more;
                    total = pieces;
                }
            }
        }
    }
    // Piece i: its tile's place in the batch (n <= 0: none) and in the scratch, its cached head, and which of the tile's pieces it is.
    __device__ __forceinline__ Place get(const Args& a, int i, int* length, int* head, int* tile, int* z) const {
        const int items = a.workgroups / a.c.heads;
        Place p{0, 0, -1, 0};
        if (per == 0) {
            *tile = i % a.workgroups;
            *z = i / a.workgroups;
            *head = *tile / items;
            p = find_place(a.b, *tile % items, a.group, 1 << shift, 1);
            p = Place{uniform(p.seq), uniform(p.begin), uniform(p.n), uniform(p.item)};
            *length = p.n > 0 ? uniform(a.b.lens[p.seq]) : 0;
            return p;
        }
        p.seq = min((int)__popcll(__ballot(upto <= i)), 63);
        const int before = p.seq > 0 ? __builtin_amdgcn_readlane(upto, p.seq - 1) : 0, many = max(__builtin_amdgcn_readlane(tiles, p.seq), 1);
        const int k = uniform((i - before) / a.c.heads);
        *head = uniform(i - before - k * a.c.heads);
        *z = uniform(k / many);
        p = place(p.seq, k - *z * many, length);
        *tile = *head * items + __builtin_amdgcn_readlane(first, p.seq) + p.item;
        return p;
    }
    __device__ __forceinline__ int walk_splits(const Args& a) const { return per ? 1 << 30 : a.splits; }
    __device__ __forceinline__ int walk_least(const Args& a) const { return per ? per : a.least; }
};

// The tiles of the many-rows kernel (not kAll), for whole waves.  Up to 64 sequences: those that there are, in front of the places that the batch has at most, and in a window what is cut is decided by
// their number.  Workgroups go round the shader engines, and fill them evenly only where none of them is empty: 8 sequences of 100 tokens, 40 heads on 8, a window of 4096, 128 tiles of at most
// 184 in two pieces each 107 us, with empty ones among them 166 (whole 159).
template <int MODE>
struct Tiles : SequenceLanes {
    int total, whole, splits;                   // tiles of all cached heads; those that are not cut; pieces of the others at most
    int each, upto;                             // tiles of a cached head (0: in their places in the batch); of this lane's sequence and those before
    __device__ __forceinline__ Tiles(const Args& a) : total(a.workgroups), whole(a.whole), splits(a.splits), each(0) {
        if (a.b.sequences > 64) return;
        read(a, 8);
        upto = SpanLanes::scan(tiles);
        each = __builtin_amdgcn_readlane(upto, 63);
        total = each * a.c.heads;
        if (MODE == kParts || splits == 1) return;
        // As the host's plan, a lane to a number of pieces.
        const int lane = threadIdx.x & 63, pieces = lane + 1, chip = tile_round(a.cus), rest = total % chip;
        const int longest = over_lanes(chunks, [](int x, int y) { return max(x, y); }), most = 0x7fffffff;
        const int time = tiles_cost(longest, pieces, rest, chip, pieces > 1 ? window_piece(total < chip) : 0);
        const bool fits = time > 0 && (pieces == 1 || (pieces <= a.splits && rest * pieces <= a.budget));
        const int cost = fits ? time : most, least = most - over_lanes(most - cost, [](int x, int y) { return max(x, y); });
        splits = __ffsll((unsigned long long)__ballot(near_least(cost, least)));
        whole = splits > 1 ? total - rest : 0;
    }
    // Tile `at`: head after head, a sequence's last tiles first.
    __device__ __forceinline__ Place get(const Args& a, int at, int* length, int* head, int* tile) const {
        const int items = a.workgroups / a.c.heads;
        if (each == 0) {
            *tile = at;
            *head = at / items;
            Place p = find_place(a.b, items - 1 - at % items, a.group, 256, 1);
            p = Place{uniform(p.seq), uniform(p.begin), uniform(p.n), uniform(p.item)};
            *length = p.n > 0 ? uniform(a.b.lens[p.seq]) : 0;
            return p;
        }
        *head = uniform(at / each);
        const int k = each - 1 - (at - *head * each), seq = min((int)__popcll(__ballot(upto <= k)), 63);
        const Place p = place(seq, k - (seq > 0 ? __builtin_amdgcn_readlane(upto, seq - 1) : 0), length);
        *tile = *head * items + items - 1 - (__builtin_amdgcn_readlane(first, seq) + p.item);
        return p;
    }
};

// Tile `at` of the many-rows kernel, and its cached head.  Causal: all heads of a tile before the next one (8 ragged prompts of up to 2500 tokens:
// 232 us, head after head 261); both ways in time: head after head (a frame of 3600 tokens, 40 heads: 5.20 ms, tile after tile 5.63).  Up to 64
// sequences: tiles with most keys first (12 ragged sequences of up to 600 tokens over caches of up to 30000: 278 us, 328 without; the prompts, whose
// lengths differ less, 232 and 227); else a sequence's last ones first.
template <int R>
__device__ __forceinline__ bool sorted_walk(const Args& a, int at, int splits, int* head, Walk* w) {
    const int items = a.workgroups / a.c.heads, item = a.causal ? at / a.c.heads : at % items;
    *head = a.causal ? at % a.c.heads : at / items;
    if (a.b.sequences < 2 || a.b.sequences > 64) return tile_walk<R>(a, items - 1 - item, splits, w);
    SpanLanes lanes(a.b, a.c.page_tokens, R, a.group);
    const int chunks = (int)(((int64_t)a.b.max_pages * a.c.page_tokens + kChunk - 1) / kChunk);
    return walk_to<R>(a, sorted_place(lanes, R, kChunk, a.causal, a.group, chunks, item), splits, w);
}

// The page of a place in the table (there is one: keys > 0), or -1: without a branch.
__device__ __forceinline__ int page_at(const Args& a, const Walk& w, int64_t place) {
    const int index = (int)min(place / a.c.page_tokens, (int64_t)a.b.max_pages - 1);
    const int page = a.b.page_table[(int64_t)w.seq * a.b.table_stride + index];
    const bool there = (place < w.keys) & ((uint32_t)page < (uint32_t)a.c.pages);
    return there ? page : -1;
}
// The same for half a chunk's page of 32 tokens in a window: one that nobody sees is not there, whatever stands beside it.
__device__ __forceinline__ int page_in_window(const Args& a, const Walk& w, const Chunks& l, int64_t place) {
    const int page = page_at(a, w, place);
    return any_seen(l, place, 32) ? page : -1;
}
// Scales of a page that page_at found.  One that is missing has 1: its codes are cleared, but a code of 0 times a scale of page 0 that is infinite or
// no number (nobody may have written that page yet) would not be 0.
__device__ __forceinline__ void page_scales(const Args& a, int page, int head, float& k, float& v) {
    const int64_t at = (int64_t)max(page, 0) * a.c.heads + head;
    const float ks = a.c.k_scale[at], vs = a.c.v_scale[at];
    k = page >= 0 ? ks : 1.0f;
    v = page >= 0 ? vs : 1.0f;
}
// Bytes of a word that holds four tokens, `left` of which exist.
__device__ __forceinline__ uint32_t tokens_left(int left) { return (uint32_t)((1ull << (8 * min(max(left, 0), 4))) - 1ull); }

// Two probabilities as they are rounded, added to a sum.  What divides a row is the sum of these: numerator and divisor then see the same roundings, and a
// dominant key's value comes out as it is.  The log-sum-exp is an fp32 result and has a sum of its own, of the probabilities before they are rounded.
__device__ __forceinline__ float add_rounded(v2bf p, float sum) {
    const v2bf ones = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(p, ones, sum, false);
}

__device__ __forceinline__ v8bf to_bf16(uint32_t lo, uint32_t hi, float scale) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Bytes of a word that stand for no finite number, as 0xff each: NaN codes, and at 2^120, the largest scale that an append sets, codes of 256 and more.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w, float scale) {
    const uint32_t t = ((w & 0x7f7f7f7fu) + (scale >= 0x1p120f ? 0x08080808u : 0x01010101u)) & 0x80808080u;     // the sign bit where the rest was 0x78 .. 0x7f, or 0x7f
    return (t >> 7) * 255u;
}
}  // namespace stream

void launch_cache_attn_tile(const stream::Args& a, hipStream_t st);
void launch_cache_attn_tile_view(const stream::Args& a, bool window, hipStream_t st);

}  // namespace dr
