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
    float *part_o, *part_ml;              // [workgroups - whole][splits][rows][D], [workgroups - whole][splits][rows][2]
    int32_t group, causal, splits, least; // query heads to a cached one; pieces at most; chunks of a piece at least
    int32_t workgroups;                   // tiles of rows of all sequences and cached heads
    int32_t whole;                        // tiles below are not cut into pieces
    float scale;                          // log2(e) / sqrt(D)
};

// The walk of a work item, in scalars: it is the same in every lane, and control flow that the compiler takes for divergent has
// cost correctness here (moves of live ranges put in front of the join's exec mask, in kernels that use most registers).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <int R>
__device__ __forceinline__ bool tile_walk(const Args& a, int item, int splits, Walk* w) {
    Place p = find_place(a.b, item, a.group, R, 1);
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

// Tile `at` of the many-rows kernel.  Causal: all heads of an item before the next one, a sequence's last items, which have most keys, first (8
// prompts of 2500 tokens: 235 us, head after head 262).  Both ways in time: head after head (a frame of 3600 tokens, 40 heads: 4.84 ms, item
// after item 4.97).
__device__ __forceinline__ void tile_of(const Args& a, int at, int* head, int* item) {
    const int items = a.workgroups / a.c.heads;
    *head = a.causal ? at % a.c.heads : at / items;
    *item = items - 1 - (a.causal ? at / a.c.heads : at % items);
}

// The page of a place in the table (there is one: keys > 0), or -1: without a branch.
__device__ __forceinline__ int page_at(const Args& a, const Walk& w, int64_t place) {
    const int index = (int)min(place / a.c.page_tokens, (int64_t)a.b.max_pages - 1);
    const int page = a.b.page_table[(int64_t)w.seq * a.b.table_stride + index];
    const bool there = (place < w.keys) & ((uint32_t)page < (uint32_t)a.c.pages);
    return there ? page : -1;
}
// Bytes of a word that holds four tokens, `left` of which exist.
__device__ __forceinline__ uint32_t tokens_left(int left) { return (uint32_t)((1ull << (8 * min(max(left, 0), 4))) - 1ull); }

__device__ __forceinline__ v8bf to_bf16(uint32_t lo, uint32_t hi, float scale) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Bytes of a word that are NaN codes, as 0xff each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    const uint32_t t = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;       // the sign bit where the rest was 0x7f
    return (t >> 7) * 255u;
}
}  // namespace stream

void launch_cache_attn_tile(const stream::Args& a, hipStream_t st);

}  // namespace dr
