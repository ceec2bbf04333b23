// Attention over the paged e4m3 cache for many rows a sequence, bf16: 256 rows (token, head of the group) to a workgroup, 64 to each of its four
// waves, one wave a SIMD.  As in k_cache_attn.hip logits are computed transposed (S^T = K Q^T, 32x32x16) and the registers of P^T
// are the second product's operand.  What differs: the codes of a chunk of 64 keys are turned into bf16 once by the workgroup
// (each wave would need all of them: converting in every wave costs as much of the vector ALU as the softmax does) and
// staged in LDS, four chunks deep, so that one barrier a chunk suffices.
//
// The fast loop takes chunks that every row sees whole.  A lone wave has to fill the matrix pipe by itself: step j (32 keys) issues the
// logits of step j + 1, the exponentials of step j and the product with the values of step j - 1, which do not depend on each other.
// Its softmax has no running maximum: the row's maximum over its first 32 keys stays the reference (2^x loses no bits, in fp32 or bf16), and
// a row whose sum leaves the range below is walked again by the plain loop, which moves its reference.  The plain loop takes the chunks
// that some rows do not see whole (the diagonal, the tail), and whatever the fast loop gave up on.
// Two sums are kept: of the probabilities as they are rounded to bf16, which divides O (see add_rounded), and of those before, for the log-sum-exp.
//
// Bound by the matrix cores and by the instructions that a lone wave issues beside them, at the power limit: 64 keys take 64 matrix instructions of 32 cycles in
// every wave, 2048 cycles of the 3700 that pass (1.83 us at the 2.0 GHz that the chip holds).  3600 rows over 72000 keys, 40 heads, d = 128: 5.0 ms, 1110 TFLOP/s
// (4 d flops a pair of a row and a key); the matrix pipes are busy for 51 %.  The rounded sum's 32 instructions are 4.5 % of that; placed elsewhere, or with their
// ones in a register, they cost the same.  Short tiles pay for their ends: of 53 us that a tile of causal prompts takes on average (15 fast chunks, 32 us) 2.7
// are its place in the batch, 3.3 its first loads, 12 the diagonal's 2.5 chunks in the plain loop, 3.5 the results; the fast loop's filling and emptying are 3.6.
// Half the rows a workgroup would let two of them overlap these, but turn every code into bf16 twice as often.
#pragma once

#include "stream_attn.h"

#include <type_traits>
#include <utility>

namespace dr {
namespace {

using namespace stream;

typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kRows = 256, kBuffers = 4;
constexpr float kRise = 8.0f;                  // of the plain loop's reference, in powers of two
constexpr float kSumMost = 1.8e19f;            // 2^64: beyond, the plain loop takes the rows again
constexpr float kScaleMost = 1.1259e15f;       // 2^50: with a page of larger values (448 * 2^50 and more) sums as large would leave fp32's range

#define DR_BARRIER() asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory")

// Whether any lane of the workgroup has x; there is a barrier between two calls.
__device__ __forceinline__ bool block_any(bool x, int (&flag)[kWaves]) {
    flag[threadIdx.x >> 6] = __ballot(x) != 0;
    DR_BARRIER();
    return uniform(flag[0] | flag[1] | flag[2] | flag[3]) != 0;
}

// Where the eight channels c (of D / 8 groups) of a key stand in its row: with 16 groups the even ones lie in front of the odd ones, so
// that the eight lanes that write a row's first halves, 16 bytes each, fall on different banks, as the lanes that read do.
template <int D>
__device__ __forceinline__ int group_place(int c) { return D == 128 ? (c >> 1) + 8 * (c & 1) : c; }

// MFMA row of a tile of 32 keys whose logits end up in register i of lane half h: 8 (i / 4) + 4 h + i % 4; token 16 h + i is put there.
__device__ __forceinline__ int row_of_token(int t) { return 8 * ((t & 15) >> 2) + 4 * (t >> 4) + (t & 3); }

// Item i of a tile's list of chunks (kWindow), or chunk i.
template <int MODE>
__device__ __forceinline__ int chunk_at(const Chunks& list, int i) {
    if constexpr (MODE == kWindow) return chunk_of(list, i);
    return i;
}

// Pages and scales of 64 chunks, one to a lane.
template <int P, int MODE>
struct Pages {
    static constexpr int SUB = P >= kChunk ? 1 : 2;
    int id[SUB];
    float ks[SUB], vs[SUB];
    __device__ __forceinline__ void fetch(const Args& a, const Walk& w, const Chunks& list, int head, int c) {
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const int64_t place = (int64_t)(MODE == kWindow ? (unsigned)chunk_of(list, c + (int)(threadIdx.x & 63)) : c + (threadIdx.x & 63)) * kChunk + 32 * s;
            id[s] = MODE == kWindow && SUB == 2 ? page_in_window(a, w, list, place) : page_at(a, w, place);
            page_scales(a, id[s], head, ks[s], vs[s]);
        }
    }
    __device__ __forceinline__ void get(int lane, int (&page)[SUB], float (&kscale)[SUB], float (&vscale)[SUB]) const {
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            page[s] = __builtin_amdgcn_readlane(id[s], lane);
            kscale[s] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks[s]), lane));
            vscale[s] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs[s]), lane));
        }
    }
};

template <int D, int P>
struct Tile {
    static constexpr int KS = D / 16, DT = D / 32, PIECES = D / 64, SUB = P >= kChunk ? 1 : 2;
    static constexpr int kKBytes = kChunk * D * 2, kStage = 2 * kKBytes;

    uint4 k[PIECES], v[PIECES];                // this thread's pieces of a chunk on their way
    float ks[SUB], vs[SUB];

    // Chunk c: its pages (valid or 0) and their scales are wave-uniform.
    __device__ __forceinline__ void load(const Args& a, int head, int c, const int (&page)[SUB], const float (&kscale)[SUB], const float (&vscale)[SUB]) {
        const int in_page = SUB == 1 ? (c * kChunk) % P : 0;
        const uint8_t *kb[SUB], *vb[SUB];      // scalars; what is left for a lane is a 32-bit offset
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const int64_t at = ((int64_t)page[s] * a.c.heads + head) * (P * D);
            kb[s] = a.c.k + at + in_page * D;
            vb[s] = a.c.v + at + in_page;
            ks[s] = kscale[s];
            vs[s] = vscale[s];
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            // piece p of the keys: 16 bytes at 16 p of the chunk; of the values: row p / 4, 16 tokens from 16 (p % 4) on
            const uint32_t p = threadIdx.x + kThreads * i, ko = 16 * p, vo = p / 4 * P + 16 * (p % 4);
            if constexpr (SUB == 1) {
                k[i] = *reinterpret_cast<const uint4*>(kb[0] + ko);
                v[i] = *reinterpret_cast<const uint4*>(vb[0] + vo);
            } else {
                if (PIECES > 1) k[i] = *reinterpret_cast<const uint4*>(kb[i] + (ko - 32 * D * i));
                else k[i] = *reinterpret_cast<const uint4*>((p < kThreads / 2 ? kb[0] : kb[SUB - 1] - 32 * D) + ko);
                v[i] = *reinterpret_cast<const uint4*>((p % 4 < 2 ? vb[0] : vb[SUB - 1] - 32) + vo);
            }
        }
    }
    // Chunk c, which is in lane `lane` of pages.  Returns a bit for each of its pages that is there.
    template <int MODE>
    __device__ __forceinline__ unsigned load(const Args& a, int head, int c, const Pages<P, MODE>& pages, int lane) {
        int page[SUB];
        float kscale[SUB], vscale[SUB];
        pages.get(lane, page, kscale, vscale);
        unsigned there = 0;
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            there |= page[s] >= 0 ? 1u << s : 0u;
            page[s] = max(page[s], 0);
        }
        load(a, head, c, page, kscale, vscale);
        return there;
    }
    // LDS addresses of this thread's halves of a piece of the keys, of the values; further pieces lie 32 rows of keys, 64 of values behind.
    static __device__ __forceinline__ void places(int base, int (&to)[4]) {
        const int p = threadIdx.x, tok = p / (D / 16), kc = p % (D / 16), r = (tok & 32) + row_of_token(tok & 31), sw = r & (D / 8 - 1);
        const int d = p / 4, vc = p % 4;
        to[0] = base + r * (2 * D) + (group_place<D>(2 * kc) ^ sw) * 16;
        to[1] = base + r * (2 * D) + (group_place<D>(2 * kc + 1) ^ sw) * 16;
        to[2] = base + kKBytes + d * (2 * kChunk) + ((2 * vc) ^ (d & 7)) * 16;
        to[3] = base + kKBytes + d * (2 * kChunk) + ((2 * vc + 1) ^ (d & 7)) * 16;
    }
    // Half x of piece j of this thread, of the keys, then of the values, into the stage `offset` bytes behind the places.
    template <int J, int X>
    __device__ __forceinline__ void store_half(const int (&to)[4], int offset) const {
        constexpr int i = J % PIECES;
        const uint4 w = J < PIECES ? k[i] : v[i];
        const bool low = J < PIECES ? (PIECES > 1 ? i == 0 : threadIdx.x < kThreads / 2) : threadIdx.x % 4 < 2;
        const float f = J < PIECES ? (SUB == 1 || low ? ks[0] : ks[SUB - 1]) : (SUB == 1 || low ? vs[0] : vs[SUB - 1]);
        const int more = J < PIECES ? i * 32 * (2 * D) : i * 64 * (2 * kChunk);
        *reinterpret_cast<__attribute__((address_space(3))) v8bf*>((__attribute__((address_space(3))) char*)(uintptr_t)(uint32_t)to[J < PIECES ? X : 2 + X] + offset + more) =
            X ? to_bf16(w.z, w.w, f) : to_bf16(w.x, w.y, f);
    }
    // Values of `left` tokens of the chunk and of the pages that are `there` count, the others are cleared; so are NaN codes: v holds 0xff in their
    // places then.  Returns whether there were any.
    __device__ __forceinline__ bool store_checked(char* stage, int left, unsigned there) {
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = threadIdx.x + kThreads * i, vc = p % 4;
            uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w}, nan[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] &= tokens_left((there >> (SUB == 1 ? 0 : vc >> 1)) & 1 ? left - 16 * vc - 4 * j : 0);
                nan[j] = nan_bytes(w[j], SUB == 1 || vc < 2 ? vs[0] : vs[SUB - 1]);
                found |= nan[j];
                w[j] &= ~nan[j];
            }
            v[i] = make_uint4(w[0], w[1], w[2], w[3]);
            store_piece(stage, i);
            v[i] = make_uint4(nan[0], nan[1], nan[2], nan[3]);
        }
        return found != 0;
    }
    __device__ __forceinline__ void store_piece(char* stage, int i) const {
        const int p = threadIdx.x + kThreads * i, tok = p / (D / 16), kc = p % (D / 16), vc = p % 4;
        const int r = (tok & 32) + row_of_token(tok & 31), sw = r & (D / 8 - 1);
        const float kf = SUB == 1 || tok < 32 ? ks[0] : ks[SUB - 1], vf = SUB == 1 || vc < 2 ? vs[0] : vs[SUB - 1];
        char* kr = stage + r * (2 * D);
        *reinterpret_cast<v8bf*>(kr + (group_place<D>(2 * kc) ^ sw) * 16) = to_bf16(k[i].x, k[i].y, kf);
        *reinterpret_cast<v8bf*>(kr + (group_place<D>(2 * kc + 1) ^ sw) * 16) = to_bf16(k[i].z, k[i].w, kf);
        store_values(stage, i, v[i], vf);
    }
    __device__ __forceinline__ void store_values(char* stage, int i, const uint4& w, float f) const {
        const int p = threadIdx.x + kThreads * i, d = p / 4, vc = p % 4;
        char* vr = stage + kKBytes + d * (2 * kChunk);
        *reinterpret_cast<v8bf*>(vr + ((2 * vc) ^ (d & 7)) * 16) = to_bf16(w.x, w.y, f);
        *reinterpret_cast<v8bf*>(vr + ((2 * vc + 1) ^ (d & 7)) * 16) = to_bf16(w.z, w.w, f);
    }
    __device__ __forceinline__ void store(char* stage) const {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) store_piece(stage, i);
    }
    // Behind store_checked: 1 where it cleared a NaN code, 0 elsewhere.
    __device__ __forceinline__ void store_cleared(char* stage) const {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) store_values(stage, i, make_uint4(v[i].x & 0x38383838u, v[i].y & 0x38383838u, v[i].z & 0x38383838u, v[i].w & 0x38383838u), 1.0f);
    }
};

template <int D>
struct Rows {
    static constexpr int KS = D / 16, DT = D / 32;
    v8bf q[2][KS];
    v16f o[2][DT];
    float m[2], l[2], div[2];                  // reference; this lane half's share of the sum, and of the rounded probabilities' sum
    int seen[2];                               // -1: no row
    int low[2];                                // kWindow: behind the sinks, what it sees begins here
};

// More wait states than a matrix instruction's result takes.
#define DR_NOPS "s_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15"
// An operation on a value that stays in its accumulation register: left to itself the compiler moves all of O to ordinary registers and back.
#define DR_IN_PLACE(op) "v_accvgpr_read_b32 %1, %0\n\ts_nop 1\n\t" op " %1, %1, %2\n\ts_nop 1\n\tv_accvgpr_write_b32 %0, %1"
template <class F>
__device__ __forceinline__ void in_place(v16f& o, F&& f) {
    asm volatile(DR_NOPS : "+a"(o));
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float x = o[j], t;
        f(x, t, j);
        o[j] = x;
    }
    asm volatile(DR_NOPS : "+a"(o));
}

// The plain loop over chunks c0 .. c1 - 1: a chunk at a time, running maximum, masks.  `pages` has the first 64.
template <int D, int P, int MODE>
__device__ __forceinline__ void walk_plain(const Args& a, const Walk& w, const Chunks& list, int head, int c0, int c1, Pages<P, MODE>& pages, char* lds, int (&flag)[kWaves],
                                           Rows<D>& r, bool busy) {
    using T = Tile<D, P>;
    const int least = seen_by(w, a.causal, a.group, w.r0);
    const int sinks = MODE == kWindow ? sink_end(a.window, w.keys) : 0;
    T t;
    unsigned coming = 0;                       // pages of the chunk on its way that are there
    auto fetch = [&](int c) {
        if (c > c0 && ((c - c0) & 63) == 0) pages.fetch(a, w, list, head, c);
        coming = t.load(a, head, chunk_at<MODE>(list, c), pages, (c - c0) & 63);
    };
    if (c0 < c1) fetch(c0);
#pragma unroll 1
    for (int at = c0; at < c1; ++at) {
        const int c = chunk_at<MODE>(list, at);
        const unsigned there = coming;
        const float slack = fmaxf(t.vs[0], t.vs[T::SUB - 1]) <= kScaleMost ? kRise : 0.0f;
        const bool whole = (MODE == kWindow ? at < full_chunks(list) : (c + 1) * kChunk <= least) && there == (1u << T::SUB) - 1;
        DR_BARRIER();                          // the last chunk is read
        // (a chunk that every row sees whole gives its NaN codes to all of them by itself)
        bool any = false;
        if (whole) {
            t.store(lds);
            DR_BARRIER();
        } else {
            any = block_any(t.store_checked(lds, w.keys - c * kChunk, there), flag);
            if (any) {
                t.store_cleared(lds + T::kStage);
                DR_BARRIER();
            }
        }
        if (at + 1 < c1) fetch(at + 1);
        if (!busy) continue;
        const int end = (c + 1) * kChunk;
        const bool masked = MODE == kWindow ? !whole : there != (1u << T::SUB) - 1 ||
                            !__all(((r.seen[0] < 0) | (r.seen[0] >= end)) & ((r.seen[1] < 0) | (r.seen[1] >= end)));
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));         // (LDS addresses are formed anew: kept, they would push O and Q out of the registers)
        const int n = lane & 31, h = lane >> 5;
        // token of logit i of tile u: 64 c + 32 u + 16 h + i; a row sees those with i below limit(qh, u)
        auto limit = [&](int qh, int u) { return (there >> (T::SUB == 1 ? 0 : u)) & 1 ? r.seen[qh] - (c * kChunk + 32 * u + 16 * h) : 0; };
        // the same as a bit for each of the 16 (kWindow)
        auto eyes = [&](int qh, int u) {
            const int base = c * kChunk + 32 * u + 16 * h;
            auto below = [&](int end) { return (1u << min(max(end - base, 0), 16)) - 1u; };
            const uint32_t bits = below(r.seen[qh]) & (~below(r.low[qh]) | below(sinks));
            return (there >> (T::SUB == 1 ? 0 : u)) & 1 ? bits : 0u;
        };
        // a tile of 32 keys at a time: logits and probabilities of a whole chunk would push O and Q out of the registers
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // (32 keys that no row of the wave sees, in a window of 1024 with 8 x 255 tokens, 128 channels: 127 us, 132 with them; 64 channels: 76, 74.5 with them)
            if (MODE == kWindow && D == 128 && masked && !__any((eyes(0, u) | eyes(1, u)) != 0)) continue;
            const int row = 32 * u + n, sw = row & (D / 8 - 1);
            v8bf kf[T::KS], vf[2][T::DT], p[2][2];
            v16f s[2];
#pragma unroll
            for (int k = 0; k < T::KS; ++k) kf[k] = *reinterpret_cast<const v8bf*>(lds + row * (2 * D) + (group_place<D>(2 * k + h) ^ sw) * 16);
            __builtin_amdgcn_sched_barrier(0);                                // (all reads on their way)
#pragma unroll
            for (int k = 0; k < T::KS; ++k)
#pragma unroll
                for (int qh = 0; qh < 2; ++qh) {
                    if (k == 0) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[qh][i] = 0.0f;
                    }
                    s[qh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], r.q[qh][k], s[qh], 0, 0, 0);
                }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < T::DT; ++i)
                    vf[k][i] = *reinterpret_cast<const v8bf*>(lds + T::kKBytes + (32 * i + n) * (2 * kChunk) + ((4 * u + 2 * h + k) ^ (n & 7)) * 16);
            __builtin_amdgcn_sched_barrier(0);
            // The reference follows the maximum once that is ahead by more than `slack`: probabilities stay below 2^slack, and O is seldom taken out
            // of the accumulation registers to be scaled.
            // (Logits into ordinary registers, whether masked or not: where a branch changes some of them, the compiler has filled the accumulation
            // registers of the other half with copies of its first element.)
            asm volatile("" : "+v"(s[0]), "+v"(s[1]));
            float ref[2], fade[2];
            bool scaled = false;
#pragma unroll
            for (int qh = 0; qh < 2; ++qh) {
                if (masked) {
                    if constexpr (MODE == kWindow) {
                        const uint32_t bits = eyes(qh, u);
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[qh][i] = (bits >> i) & 1u ? s[qh][i] : -INFINITY;
                    } else {
                        const int lim = limit(qh, u);
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[qh][i] = i < lim ? s[qh][i] : -INFINITY;
                    }
                }
                float top = s[qh][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) top = fmaxf(top, s[qh][i]);
                top = fmaxf(top, __shfl_xor(top, 32)) * a.scale;
                const bool rise = top > r.m[qh] + slack;
                const float now = rise ? top : r.m[qh];
                ref[qh] = now == -INFINITY ? 0.0f : now;
                fade[qh] = rise ? __builtin_amdgcn_exp2f(r.m[qh] - ref[qh]) : 1.0f;
                scaled = scaled | (rise & (r.m[qh] != -INFINITY));                   // (a row without keys so far has sums of 0)
                r.m[qh] = now;
            }
            if (__any(scaled)) {
#pragma unroll
                for (int qh = 0; qh < 2; ++qh) {
                    r.l[qh] *= fade[qh];
                    r.div[qh] *= fade[qh];
#pragma unroll
                    for (int i = 0; i < T::DT; ++i) in_place(r.o[qh][i], [&](float& x, float& t, int) { asm volatile(DR_IN_PLACE("v_mul_f32") : "+a"(x), "=&v"(t) : "v"(fade[qh])); });
                }
            }
#pragma unroll
            for (int qh = 0; qh < 2; ++qh) {
                float more = 0.0f, more_div = 0.0f;                            // (a tile's: added one by one, small ones would be lost beside a large sum)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(s[qh][8 * k + j], a.scale, -ref[qh]));
                        p[qh][k][j] = (__bf16)e;
                        more += e;
                        if (j & 1) more_div = add_rounded(v2bf{p[qh][k][j - 1], p[qh][k][j]}, more_div);
                    }
                r.l[qh] += more;
                r.div[qh] += more_div;
            }
#pragma unroll
            for (int i = 0; i < T::DT; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int qh = 0; qh < 2; ++qh) r.o[qh][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k][i], p[qh][k], r.o[qh][i], 0, 0, 0);
        }
        if (any) {                             // NaN codes for the rows that see them: a probability of 0 would not have silenced them
#pragma unroll
            for (int i = 0; i < T::DT; ++i)
#pragma unroll
                for (int qh = 0; qh < 2; ++qh) {
                    v16f hit;
#pragma unroll
                    for (int j = 0; j < 16; ++j) hit[j] = 0.0f;
#pragma unroll 1
                    for (int uk = 0; uk < 4; ++uk) {
                        v8bf eye;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const bool sees = MODE == kWindow ? (eyes(qh, uk >> 1) >> (8 * (uk & 1) + j)) & 1u : 8 * (uk & 1) + j < limit(qh, uk >> 1);
                            eye[j] = (__bf16)(sees ? 1.0f : 0.0f);
                        }
                        const v8bf bad = *reinterpret_cast<const v8bf*>(lds + T::kStage + T::kKBytes + (32 * i + n) * (2 * kChunk) + ((4 * (uk >> 1) + 2 * h + (uk & 1)) ^ (n & 7)) * 16);
                        hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bad, eye, hit, 0, 0, 0);
                    }
                    in_place(r.o[qh][i], [&](float& x, float& t, int j) { asm volatile(DR_IN_PLACE("v_add_f32") : "+a"(x), "=&v"(t) : "v"(hit[j] > 0.0f ? NAN : 0.0f)); });
                }
        }
    }
    DR_BARRIER();
}

// Matrix instructions of the fast loop go through inline assembly: logits live in ordinary registers (the exponentials read them), O and Q in
// accumulation registers (left to itself the compiler puts all results there and copies the logits back, 64 moves a chunk).  The
// compiler then does not know what these are: whoever reads a result with the vector ALU is kept half a step behind by the schedule,
// and in front of the loop and behind it the wave waits.
__device__ __forceinline__ void mfma_s0(v16f& s, const v8bf& k, const v8bf& q) { asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "a"(q)); }
__device__ __forceinline__ void mfma_s(v16f& s, const v8bf& k, const v8bf& q) { asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q)); }
__device__ __forceinline__ void mfma_o(v16f& o, const v8bf& v, const v8bf& p) { asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(v), "v"(p)); }

template <class F, int... I>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F&& f) { (f(std::integral_constant<int, I>{}), ...); }

// The fast loop over chunks c0 .. c1 - 1 (two at least, on their way in t0 and t1), all of them seen whole by every row.  Its four passes are not left in between: behind
// the last chunk it takes that again with exponents of -infinity.  Returns whether a page was missing or too large.
template <int D, int P, int MODE>
__device__ __forceinline__ bool walk_fast(const Args& a, const Walk& w, const Chunks& list, int head, int c0, int c1, const Tile<D, P>& t0, const Tile<D, P>& t1, char* lds,
                                          Rows<D>& r, bool busy) {
    using T = Tile<D, P>;
    constexpr int SUB = T::SUB, FRAGS = T::KS + 2 * T::DT, SLOTS = 2 * FRAGS, EACH = 32 / SLOTS, AHEAD = 4;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    int zero;
    asm volatile("v_mov_b32 %0, 0" : "=v"(zero));       // page numbers and scales go through vector loads: scalar ones would share the LDS reads' counter
    bool missing = false;
    T t;
    int id[SUB];
    auto real = [&](int c) { return MODE != kWindow || c < list.full0 ? c : c - list.full0 + list.at1; };      // (the list's first part, see Chunks)
    auto number = [&](int c) {                  // page numbers of chunk c (past the end: of the last one again)
        const int at = (int)((int64_t)real(min(c, c1 - 1)) * kChunk / P) + zero;
#pragma unroll
        for (int s = 0; s < SUB; ++s) id[s] = a.b.page_table[(int64_t)w.seq * a.b.table_stride + at + s];
    };
    auto fetch = [&](int c) {                   // chunk c, whose page numbers are in id
        c = min(c, c1 - 1);
        int page[SUB];
        float ks[SUB], vs[SUB];
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            page[s] = __builtin_amdgcn_readfirstlane(id[s]);
            missing = missing || (uint32_t)page[s] >= (uint32_t)a.c.pages;
            page[s] = (uint32_t)page[s] < (uint32_t)a.c.pages ? page[s] : 0;
            const int64_t at = (int64_t)page[s] * a.c.heads + head + zero;
            ks[s] = a.c.k_scale[at];
            vs[s] = a.c.v_scale[at];
        }
        t.load(a, head, real(c), page, ks, vs);
    };
    // Addresses of the operands in stages 0 and 1, and in stages 2 and 3 (an instruction's offset has 16 bits)
    int kaddr[2][T::KS], vaddr[2][4], to[2][4];
    const int base = (int)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int k = 0; k < T::KS; ++k) kaddr[x][k] = base + 2 * x * T::kStage + n * (2 * D) + (group_place<D>(2 * k + h) ^ (n & (D / 8 - 1))) * 16;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            vaddr[x][k] = base + 2 * x * T::kStage + T::kKBytes + n * (2 * kChunk) + ((4 * (k >> 1) + 2 * h + (k & 1)) ^ (n & 7)) * 16;
        T::places(base + 2 * x * T::kStage, to[x]);
    }
    float ref[2], sum[2][4] = {}, div[2] = {};

    number(c0 + 2);
    DR_BARRIER();
    t0.store(lds);
    t1.store(lds + T::kStage);
    for (int i = threadIdx.x; i < T::kKBytes / 16; i += kThreads) *reinterpret_cast<uint4*>(lds + 3 * T::kStage + T::kKBytes + 16 * i) = uint4{0, 0, 0, 0};
    fetch(c0 + 2);
    number(c0 + 3);
    DR_BARRIER();

    if (!busy) {                                // a wave without rows: its share of the chunks, and the barriers
#pragma unroll 1
        for (int c = c0; c < c0 + ((c1 - c0 + 3) & ~3); ++c) {
            DR_BARRIER();
            t.store(lds + ((c + 2 - c0) & 3) * T::kStage);
            fetch(c + 3);
            number(c + 4);
        }
        DR_BARRIER();
        DR_BARRIER();
        return missing;
    }

    v16f s[2][2];                               // [step parity][query half]
    typedef uint32_t v4u __attribute__((ext_vector_type(4)));
    v4u p[2][2][2];                             // [step parity][query half][16 keys]
#pragma unroll
    for (int qh = 0; qh < 2; ++qh)
#pragma unroll
        for (int k = 0; k < 2; ++k) p[1][qh][k] = v4u{0, 0, 0, 0};

    typedef __attribute__((address_space(3))) const v8bf* lds_v8;
    typedef __attribute__((address_space(3))) const char* lds_c;
    // Operand f of a step: keys of tile kt of stage ks for f < KS, then values of tile vt of stage vs
    auto read = [&](int f, int ks, int kt, int vs, int vt) {
        if (f < T::KS) return *reinterpret_cast<lds_v8>((lds_c)(uintptr_t)(uint32_t)kaddr[ks >> 1][f] + (ks & 1) * T::kStage + kt * (32 * 2 * D));
        const int k = (f - T::KS) / T::DT, i = (f - T::KS) % T::DT;
        return *reinterpret_cast<lds_v8>((lds_c)(uintptr_t)(uint32_t)vaddr[vs >> 1][2 * vt + k] + (vs & 1) * T::kStage + i * (32 * 2 * kChunk));
    };
    v8bf fr[AHEAD];
    // One step: logits of the next tile into s[1 - E], exponentials of s[E] into p[E], products of p[1 - E] with the tile before.  A slot is
    // a matrix instruction with EACH exponentials in its shadow; operands are read three operands (six slots) ahead.  Step A (E = 0) of the chunk
    // in stage X takes its tile 1 and the values of tile 1 of the chunk before; step B tile 0 of the next chunk and the values of its own tile 0.
    // A lone wave pays some 4.5 cycles for every instruction beyond the five that the matrix instruction covers: stages are
    // constants (four passes to a loop), lane addresses have no additions.
    auto step = [&](auto parity, auto stage, int c) {
        if (decltype(parity)::value == 0) {
            ref[0] = c < c1 ? ref[0] : -INFINITY;
            ref[1] = c < c1 ? ref[1] : -INFINITY;
        }
        constexpr int E = decltype(parity)::value, X = decltype(stage)::value;
        constexpr int prev = (X + 3) & 3, next = (X + 1) & 3, free = (X + 2) & 3;
        const int ks = E ? next : X, vs = E ? X : prev;
        // Neighbouring instructions do not wait for each other: an exponent is formed before the exponential of the one in front of it, probabilities
        // are summed and packed a place behind theirs.
        float w0 = 0.0f, w1 = 0.0f, x = fmaf(s[E][0][0], a.scale, ref[0]);
        auto used = [&](int e) {                         // probability e is w1
            sum[e / 16][e & 3] += w1;
            if (e & 1) {
                const v2bf pair = {(__bf16)w0, (__bf16)w1};
                uint32_t bits = __builtin_bit_cast(uint32_t, pair);
                div[e / 16] = add_rounded(pair, div[e / 16]);
                asm volatile("" : "+v"(bits));           // (here, not where the last pair of a fragment is)
                p[E][e / 16][e / 8 % 2][e % 8 / 2] = bits;
            }
        };
        auto slot = [&](auto number_of) {
            constexpr int i = decltype(number_of)::value, f = i / 2, qh = i & 1;
            if (f < T::KS) {
                if (f == 0) mfma_s0(s[1 - E][qh], fr[f % AHEAD], r.q[qh][f < T::KS ? f : 0]);
                else mfma_s(s[1 - E][qh], fr[f % AHEAD], r.q[qh][f < T::KS ? f : 0]);
            } else {
                mfma_o(r.o[qh][(f - T::KS + T::DT * 2) % T::DT], fr[f % AHEAD], __builtin_bit_cast(v8bf, p[1 - E][qh][(f >= T::KS ? f - T::KS : 0) / T::DT]));
            }
            if (qh == 0) {                      // the operand before this slot's is used up
                constexpr int g = f - 1 + AHEAD;
                fr[g % AHEAD] = g < FRAGS ? read(g, ks, 1 - E, vs, 1 - E) : read(g - FRAGS, next, E, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int e = i * EACH + j;
                const float v = __builtin_amdgcn_exp2f(x);
                if (e < 31) x = fmaf(s[E][(e + 1) / 16 & 1][(e + 1) % 16], a.scale, ref[(e + 1) / 16 & 1]);
                if (e > 0) used(e - 1);
                w0 = w1;
                w1 = v;
            }
            if (E == 0 && i == SLOTS / 4) {
                // chunk c + 1 was written in the last pass; three reads since then may be on their way (D = 64: there were no more)
                asm volatile("s_waitcnt lgkmcnt(3)\n\ts_barrier" ::: "memory");
            }
            if (E == 1) {
                constexpr int PER = SLOTS / (4 * T::PIECES);       // half a piece every so many slots
                if constexpr (i % PER == PER / 2) t.template store_half<i / PER / 2, i / PER % 2>(to[free >> 1], (free & 1) * T::kStage);
                if (i == SLOTS - 1) {
                    missing = missing | !(fmaxf(t.vs[0], t.vs[SUB - 1]) <= kScaleMost);
                    fetch(c + 3);
                    number(c + 4);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        each(std::make_integer_sequence<int, SLOTS>{}, slot);
        used(31);
        __builtin_amdgcn_sched_barrier(0);
    };
    v8bf first[T::KS];
    // Q and O go into accumulation registers here, and are there before the first instruction that the compiler does not know: it would
    // neither wait for a load into them nor leave room behind a move (both have given wrong logits).
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int k = 0; k < T::KS; ++k) asm volatile("s_nop 7" : "+a"(r.q[0][k]), "+a"(r.q[1][k]));
#pragma unroll
    for (int i = 0; i < T::DT; ++i) asm volatile("s_nop 7" : "+a"(r.o[0][i]), "+a"(r.o[1][i]));
#pragma unroll
    for (int k = 0; k < T::KS; ++k) first[k] = read(k, 0, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < T::KS; ++k)
#pragma unroll
        for (int qh = 0; qh < 2; ++qh) {
            if (k == 0) mfma_s0(s[0][qh], first[k], r.q[qh][k]);
            else mfma_s(s[0][qh], first[k], r.q[qh][k]);
        }
    asm volatile(DR_NOPS : "+v"(s[0][0]), "+v"(s[0][1]));
#pragma unroll
    for (int qh = 0; qh < 2; ++qh) {            // the reference: the maximum over the first 32 keys
        float top = s[0][qh][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[0][qh][i]);
        top = fmaxf(top, __shfl_xor(top, 32)) * a.scale;
        missing = missing | !(fabsf(top) < INFINITY);
        r.m[qh] = top;
        ref[qh] = -top;
    }
#pragma unroll
    for (int f = 0; f < AHEAD - 1; ++f) fr[f] = read(f, 0, 1, 0, 0);
    fr[AHEAD - 1] = first[0];                   // (read in the first slot)
    __builtin_amdgcn_sched_barrier(0);
    // The first products take the values of a chunk that is not there: stage 3 is cleared for them.
    auto pass = [&](auto stage, int c) {
        step(std::integral_constant<int, 0>{}, stage, c);
        step(std::integral_constant<int, 1>{}, stage, c);
    };
#pragma unroll 1
    for (int c = c0; c < c1; c += 4) {
        pass(std::integral_constant<int, 0>{}, c);
        pass(std::integral_constant<int, 1>{}, c + 1);
        pass(std::integral_constant<int, 2>{}, c + 2);
        pass(std::integral_constant<int, 3>{}, c + 3);
        // (the sums of four chunks: added one by one, small probabilities would be lost beside a large sum)
#pragma unroll
        for (int qh = 0; qh < 2; ++qh) {
            r.l[qh] += (sum[qh][0] + sum[qh][1]) + (sum[qh][2] + sum[qh][3]);
            r.div[qh] += div[qh];
            sum[qh][0] = sum[qh][1] = sum[qh][2] = sum[qh][3] = div[qh] = 0.0f;
        }
    }
    DR_BARRIER();
    v8bf last[2][T::DT];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < T::DT; ++i)
            last[k][i] = *reinterpret_cast<lds_v8>((lds_c)(uintptr_t)(uint32_t)vaddr[1][2 + k] + T::kStage + i * (32 * 2 * kChunk));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < T::DT; ++i)
#pragma unroll
            for (int qh = 0; qh < 2; ++qh) mfma_o(r.o[qh][i], last[k][i], __builtin_bit_cast(v8bf, p[1][qh][k]));
    if constexpr (T::DT == 4)
        asm volatile(DR_NOPS : "+a"(r.o[0][0]), "+a"(r.o[1][0]), "+a"(r.o[0][1]), "+a"(r.o[1][1]), "+a"(r.o[0][2]), "+a"(r.o[1][2]), "+a"(r.o[0][3]), "+a"(r.o[1][3]));
    else
        asm volatile(DR_NOPS : "+a"(r.o[0][0]), "+a"(r.o[1][0]), "+a"(r.o[0][1]), "+a"(r.o[1][1]));
    DR_BARRIER();
    return missing;
}

struct NoTiles {};
template <int MODE>
__device__ __forceinline__ auto tiles_of(const Args& a) {
    if constexpr (MODE == kAll) return NoTiles{}; else return Tiles<MODE>(a);
}

template <int D, int P, int MODE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void k_cache_attn_tile(const Args a) {
    using T = Tile<D, P>;
    __shared__ __align__(16) char lds[kBuffers * T::kStage];     // (as large as 256 rows of fp32 results)
    __shared__ float4 s_sums[kRows];
    __shared__ int flag[kWaves];
    // The last tiles, which would leave compute units idle, are cut into pieces of their key range.  Workgroups go round the eight XCDs: both
    // ways in time each takes consecutive tiles, which are mostly of one head and read the same keys at the same time.
    int whole = a.whole, rest = a.workgroups - a.whole, most = a.splits;
    const auto tiles = tiles_of<MODE>(a);
    if constexpr (MODE != kAll) {
        whole = tiles.whole;
        rest = tiles.total - whole;
        most = tiles.splits;
    }
    const int pieces = rest * most, i = (int)blockIdx.x - whole;
    int j = i < 0 ? (int)blockIdx.x : i;
    if (MODE != kAll && i >= (pieces + 7) / 8 * 8) return;
    if (MODE != kAll || !a.causal) j = i < 0 ? j % 8 * (whole / 8) + j / 8 : j % 8 * ((pieces + 7) / 8) + j / 8;
    if (i >= 0 && j >= pieces) return;
    const int z = i < 0 ? 0 : j / rest, at = i < 0 ? j : whole + j % rest, splits = i < 0 ? 1 : most;
    int head;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
    Walk w;
    Chunks list;
    int tile = at - whole;             // its place in the scratch
    if constexpr (MODE == kAll) {
        if (!sorted_walk<kRows>(a, at, splits, &head, &w)) return;
    } else {
        int len, place;
        const Place p = tiles.get(a, at, &len, &head, &place);
        bool any;
        if constexpr (MODE == kWindow) {
            any = window_walk_to(a, kRows, p, len, splits, a.least, &w, &list);
        } else {
            tile = place;
            any = known_walk_to(a, kRows, p, len, splits, a.least, &w);
        }
        if (!any) return;
    }
    if (z >= max(w.active, 1)) return;
    const int c0 = z * w.per, c1 = min(c0 + w.per, w.chunks);

    Rows<D> r;
    const Rows256 split = uniform_rows(w.r0, a.group);
    const int rows = min(kRows, w.rows - w.r0);
    const bool busy = 64 * wave < rows;
#pragma unroll
    for (int qh = 0; qh < 2; ++qh) {
        const int row = 64 * wave + 32 * qh + n;
        const bool there = row < rows;
        int token, hd;
        row_at(split, there ? row : 0, &token, &hd);
        if constexpr (MODE == kWindow) {
            const Reach x = reach_at(a.window, w.keys, w.shift + token);
            r.seen[qh] = there ? x.hi : -1;
            r.low[qh] = x.lo;
        } else {
            r.seen[qh] = there ? seen_at(w, a.causal, token) : -1;
        }
        const char* src = a.q + (int64_t)(w.begin + token) * a.qt + (int64_t)(head * a.group + hd) * a.qh;
#pragma unroll
        for (int k = 0; k < T::KS; ++k) r.q[qh][k] = *reinterpret_cast<const v8bf*>(src + (16 * k + 8 * h) * 2);
    }
    const int full = min(MODE == kWindow ? full_chunks(list) : seen_at(w, a.causal, split.token) / kChunk, c1);          // chunks below are seen whole by every row
    auto clear = [&] {
#pragma unroll
        for (int qh = 0; qh < 2; ++qh) {
            r.m[qh] = -INFINITY;
            r.l[qh] = r.div[qh] = 0.0f;
#pragma unroll
            for (int i = 0; i < T::DT; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) r.o[qh][i][j] = 0.0f;
        }
    };
    clear();
    // Chunks of the fast loop: a pass of four, some of them empty, costs as much as two in the plain loop (1.9 and 4.1 us a chunk on a full chip).
    int from = c0, fast = full - c0;
    if ((fast & 3) == 1) --fast;
    const int end = c0 + fast;
    Pages<P, MODE> pages{};
    if (c0 < c1) pages.fetch(a, w, list, head, c0);    // (without keys the table may have no entry)
    if (fast > 2) {
        T t0, t1;
        const unsigned there = t0.load(a, head, chunk_at<MODE>(list, c0), pages, 0) & t1.load(a, head, chunk_at<MODE>(list, c0 + 1), pages, 1);
        pages.fetch(a, w, list, head, end);           // those behind the fast loop
        bool again = there != (1u << T::SUB) - 1 || !(fmaxf(fmaxf(t0.vs[0], t0.vs[T::SUB - 1]), fmaxf(t1.vs[0], t1.vs[T::SUB - 1])) <= kScaleMost);
        if (!block_any(again, flag)) {
            again = walk_fast<D, P, MODE>(a, w, list, head, c0, end, t0, t1, lds, r, busy);
#pragma unroll
            for (int qh = 0; qh < 2; ++qh) again = again | ((r.seen[qh] > 0) & !(r.l[qh] <= kSumMost));
            from = end;
            if (block_any(again, flag)) {
                clear();
                from = c0;
            }
        }
        if (from != end) pages.fetch(a, w, list, head, from);
    }
    walk_plain<D, P, MODE>(a, w, list, head, from, c1, pages, lds, flag, r, busy);

    // Results go through LDS: whole rows to memory, and no branch while they fill the registers.
    const bool last = MODE != kParts && w.active <= 1;
#pragma unroll
    for (int qh = 0; qh < 2; ++qh) {
        const int row = 64 * wave + 32 * qh + n;
        const float total = r.l[qh] + __shfl_xor(r.l[qh], 32), divisor = r.div[qh] + __shfl_xor(r.div[qh], 32);
        const float inv = last ? 1.0f / (divisor == 0.0f ? 1.0f : divisor) : 1.0f;
        s_sums[row] = make_float4(r.m[qh], total, divisor, 0.0f);
        // a lane holds channels 32 i + 8 g + 4 h + 0..3 of its row
#pragma unroll
        for (int i = 0; i < T::DT; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c4 = 8 * i + 2 * g + h;
                const float y0 = r.o[qh][i][4 * g] * inv, y1 = r.o[qh][i][4 * g + 1] * inv, y2 = r.o[qh][i][4 * g + 2] * inv, y3 = r.o[qh][i][4 * g + 3] * inv;
                const v2bf lo = {(__bf16)y0, (__bf16)y1}, hi = {(__bf16)y2, (__bf16)y3};
                // (16 bytes of a row swapped by its number: the 32 rows of a wave would fall on the same banks)
                if (last) *reinterpret_cast<uint2*>(lds + row * (2 * D) + ((c4 >> 1) ^ (row & (D / 8 - 1))) * 16 + (c4 & 1) * 8) =
                    make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
                else *reinterpret_cast<float4*>(lds + row * (4 * D) + (c4 ^ (row & (D / 4 - 1))) * 16) = make_float4(y0, y1, y2, y3);
            }
    }
    __syncthreads();
    if (last) {
        constexpr int C = D / 8;                // pieces of 16 bytes
        for (int j = threadIdx.x; j < rows * C; j += kThreads) {
            const int row = j / C, c = j % C;
            int token, hd;
            row_at(split, row, &token, &hd);
            *reinterpret_cast<uint4*>(a.o + (int64_t)(w.begin + token) * a.ot + (int64_t)(head * a.group + hd) * a.oh + c * 16) =
                *reinterpret_cast<const uint4*>(lds + row * (2 * D) + (c ^ (row & (D / 8 - 1))) * 16);
        }
        if (a.lse && threadIdx.x < rows) {
            int token, hd;
            row_at(split, threadIdx.x, &token, &hd);
            const float m = s_sums[threadIdx.x].x, total = s_sums[threadIdx.x].y;
            a.lse[(int64_t)(head * a.group + hd) * a.b.tokens + w.begin + token] = total == 0.0f ? -INFINITY : (m == -INFINITY ? 0.0f : m) * kLn2 + logf(total);
        }
    } else {
        constexpr int C = D / 4;
        const int64_t slot = ((int64_t)(MODE == kAll ? at - a.whole : tile) * (MODE == kWindow ? most : a.splits) + z) * kRows;
        for (int j = threadIdx.x; j < rows * C; j += kThreads) {
            const int row = j / C, c = j % C;
            *reinterpret_cast<float4*>(a.part_o + (slot + row) * D + 4 * c) = *reinterpret_cast<const float4*>(lds + row * (4 * D) + (c ^ (row & (D / 4 - 1))) * 16);
        }
        if (threadIdx.x < rows) a.part_sums[slot + threadIdx.x] = s_sums[threadIdx.x];
    }
}

template <int MODE>
void launch_tile(const Args& a, hipStream_t st) {
    int64_t pieces = (int64_t)(a.workgroups - a.whole) * a.splits, whole = a.whole;
    if (MODE == kWindow && a.splits > 1 && a.b.sequences <= 64) {       // (as many as Tiles may make of it)
        whole = a.workgroups / tile_round(a.cus) * tile_round(a.cus);
        pieces = a.budget;
    }
    const unsigned grid = (unsigned)(whole + (pieces + 7) / 8 * 8);
    if (a.c.d == 128) {
        if (a.c.page_tokens == 128) k_cache_attn_tile<128, 128, MODE><<<grid, kThreads, 0, st>>>(a);
        else if (a.c.page_tokens == 64) k_cache_attn_tile<128, 64, MODE><<<grid, kThreads, 0, st>>>(a);
        else k_cache_attn_tile<128, 32, MODE><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (a.c.page_tokens == 128) k_cache_attn_tile<64, 128, MODE><<<grid, kThreads, 0, st>>>(a);
        else if (a.c.page_tokens == 64) k_cache_attn_tile<64, 64, MODE><<<grid, kThreads, 0, st>>>(a);
        else k_cache_attn_tile<64, 32, MODE><<<grid, kThreads, 0, st>>>(a);
    }
}

}  // namespace
}  // namespace dr
