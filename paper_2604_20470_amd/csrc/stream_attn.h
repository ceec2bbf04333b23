// What the kernels of the attention over the paged cache share.  Internal: not part of the public ABI.
#pragma once

#include "stream_common.h"

namespace dr {
namespace stream {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4, kChunk = 64;
constexpr float kLn2 = 0.69314718055994530942f;

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

}  // namespace dr
