// Softmax attention of new tokens over the paged e4m3 cache.
//
// One pass over the keys with the running maximum and sum of the softmax.  Rows are (token, head) pairs of one cached head, so the heads that share
// keys share their loads.  The logits are computed transposed, S^T = K Q^T: a lane then holds one row's logits, row statistics need no
// broadcast, and the registers of P^T are the second product's operand as they are: which key sits in which matrix row is free, and is
// chosen such that a lane group's logits belong to consecutive tokens, whose V codes lie side by side in the page (tokens
// innermost).  Codes go from memory to registers, are turned into bf16 there (exactly; the page's power of two is applied by the same
// instruction), and meet Q and P on the matrix cores.
// Bound by memory: a single row of two sequences of 264000 keys, 24 heads, d = 128: 550 us, 5.9 TB/s of codes; 48 ragged sequences of up to 16384 keys,
// five rows to a cached head, 80 us where a copy's rate gives 51 (the pieces' ends; 71 us on inputs that the last-level cache still holds).  Two workgroups stay on a compute unit, one waits for its
// loads while the other computes.  In fp32 the three parts of queries and of probabilities make it three matrix instructions for one.
#include "stream_attn.h"

namespace dr {
namespace {

using namespace stream;

// x as PARTS bf16 that add up to it (to 8 bits, 16, or all 24).
template <int PARTS>
__device__ __forceinline__ void split(const float (&x)[8], v8bf (&p)[PARTS]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float rest = x[j];
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
            p[k][j] = (__bf16)rest;
            if (k + 1 < PARTS) rest -= (float)p[k][j];
        }
    }
}
__device__ __forceinline__ v8bf ones_where(uint32_t lo, uint32_t hi) {        // 1 for a byte 0xff, 0 for 0
    v8bf r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = (__bf16)((((j < 4 ? lo : hi) >> (8 * (j & 3))) & 1u) ? 1.0f : 0.0f);
    return r;
}

// 16 * NR rows of a tile; the four waves take the chunks of a piece in turn and join their sums at its end.
template <typename T, int D, int P, int NR>
__global__ __launch_bounds__(kThreads, 2) void k_cache_attn_rows(const Args a) {
    // Parts of a query, and of a probability: all 24 bits in fp32; bf16 queries are whole, and probabilities keep 16 bits where the rows are few and the
    // matrix cores wait for memory anyway
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, PROBS = sizeof(T) == 4 ? 3 : NR == 1 ? 2 : 1, R = 16 * NR, KS = D / 64, DT = D / 16, SUB = P >= kChunk ? 1 : 2;
    __shared__ float s_sums[NR][kWaves][16][3];
    __shared__ __align__(16) float s_o[NR][kWaves][16][D + 4];
    const int items = a.workgroups / a.c.heads, head = blockIdx.x / items, item = blockIdx.x % items, z = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, h4 = lane >> 4;
    Walk w;
    if (!tile_walk<R>(a, item, a.splits, &w)) return;
    if (z >= max(w.active, 1)) return;
    const int c0 = z * w.per, c1 = min(c0 + w.per, w.chunks);

    v8bf q[NR][2 * KS][PARTS];
    int seen[NR];
    const Rows256 places = uniform_rows(w.r0, a.group);
    const int least = seen_at(w, a.causal, places.token);                     // of all rows of the tile
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = w.r0 + 16 * r + n;
        const bool there = row < w.rows;
        int token, hd;
        row_at(places, there ? 16 * r + n : 0, &token, &hd);
        seen[r] = there ? seen_at(w, a.causal, token) : 0;
        const char* at = a.q + (int64_t)(w.begin + token) * a.qt + (int64_t)(head * a.group + hd) * a.qh;
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t) {
            const int ch = 64 * (t >> 1) + 16 * h4 + 8 * (t & 1);
            float x[8];
            if constexpr (PARTS == 1) {
                Pack<T>::load(at + ch * sizeof(T), x);
            } else {
                float y[4], v[4];
                Pack<T>::load(at + ch * sizeof(T), y);
                Pack<T>::load(at + (ch + 4) * sizeof(T), v);
#pragma unroll
                for (int j = 0; j < 4; ++j) { x[j] = y[j]; x[4 + j] = v[j]; }
            }
            if (!there) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = 0.0f;
            }
            split<PARTS>(x, q[r][t]);
        }
    }
    v4f acc[NR][DT];
    float m[NR], l[NR], div[NR];              // reference, sum, sum of the rounded probabilities (with several parts: the sum itself)
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        m[r] = -INFINITY;
        l[r] = div[r] = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[r][i] = v4f{0, 0, 0, 0};
    }

    const int64_t tile_bytes = (int64_t)P * D;
    int ids[SUB];
    float ksc[SUB], vsc[SUB];                                                 // lane i: of the wave's i-th chunk from here on
    for (int c = c0 + wave, it = 0; c < c1; c += kWaves, ++it) {
        if ((it & 63) == 0) {
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const int64_t place = (int64_t)(c + kWaves * lane) * kChunk + 32 * s;
                const int page = page_at(a, w, place);
                ids[s] = page;
                page_scales(a, page, head, ksc[s], vsc[s]);
            }
        }
        int page[SUB];
        float ks[SUB], vs[SUB];
        bool whole = (c + 1) * kChunk <= least;                               // every row sees all of the chunk
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            page[s] = __builtin_amdgcn_readlane(ids[s], it & 63);
            ks[s] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc[s]), it & 63));
            vs[s] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc[s]), it & 63));
            whole = whole && page[s] >= 0;
        }
        const int in_page = SUB == 1 ? (c * kChunk) % P : 0;
        uint4 kq[4][KS];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int s = SUB == 1 ? 0 : u >> 1;
            const int tok = SUB == 1 ? in_page + 16 * (n >> 2) + 4 * u + (n & 3) : 8 * (n >> 2) + 4 * (u & 1) + (n & 3);
            const uint8_t* at = a.c.k + ((int64_t)max(page[s], 0) * a.c.heads + head) * tile_bytes + tok * D + 16 * h4;
#pragma unroll
            for (int t = 0; t < KS; ++t) kq[u][t] = *reinterpret_cast<const uint4*>(at + 64 * t);
        }
        uint32_t vw[DT][4];
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const int64_t row = (16 * i + n) * P;
            if constexpr (SUB == 1) {
                const uint4 x = *reinterpret_cast<const uint4*>(a.c.v + ((int64_t)max(page[0], 0) * a.c.heads + head) * tile_bytes + row + in_page + 16 * h4);
                vw[i][0] = x.x; vw[i][1] = x.y; vw[i][2] = x.z; vw[i][3] = x.w;
            } else {
#pragma unroll
                for (int s = 0; s < SUB; ++s) {
                    const uint2 x = *reinterpret_cast<const uint2*>(a.c.v + ((int64_t)max(page[s], 0) * a.c.heads + head) * tile_bytes + row + 8 * h4);
                    vw[i][2 * s] = x.x; vw[i][2 * s + 1] = x.y;
                }
            }
        }
        // token of logit (u, i) of this lane: 4 of them for each u
        auto token = [&](int u) { return c * kChunk + (SUB == 1 ? 16 * h4 + 4 * u : 32 * (u >> 1) + 8 * h4 + 4 * (u & 1)); };
        v8bf p[NR][2][PROBS];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            v4f s[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                s[u] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < KS; ++t) {
                    const float f = ks[SUB == 1 ? 0 : u >> 1];
                    const v8bf lo = to_bf16(kq[u][t].x, kq[u][t].y, f), hi = to_bf16(kq[u][t].z, kq[u][t].w, f);
#pragma unroll
                    for (int k = PARTS - 1; k >= 0; --k) {
                        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, q[r][2 * t][k], s[u], 0, 0, 0);
                        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q[r][2 * t + 1][k], s[u], 0, 0, 0);
                    }
                }
            }
            if (!whole) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const bool page_there = page[SUB == 1 ? 0 : u >> 1] >= 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((token(u) + i < seen[r]) & page_there)) s[u][i] = -INFINITY;
                }
            }
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][i]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(m[r], top * a.scale), ref = now == -INFINITY ? 0.0f : now;
            const float fade = __builtin_amdgcn_exp2f(m[r] - ref);             // (0 for the first keys of a row: its sums are 0 as well)
            m[r] = now;
            l[r] *= fade;
            if constexpr (PROBS == 1) div[r] *= fade;
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[r][i] *= fade;
            float more = 0.0f;                                                 // (a chunk's: added one by one, small ones would be lost beside a large sum)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    e[j] = __builtin_amdgcn_exp2f(fmaf(s[2 * k + (j >> 2)][j & 3], a.scale, -ref));
                    more += e[j];
                }
                split<PROBS>(e, p[r][k]);
                if constexpr (PROBS == 1) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) div[r] = add_rounded(v2bf{p[r][k][0][j], p[r][k][0][j + 1]}, div[r]);
                }
            }
            l[r] += more;
        }
        // A probability of 0 does not silence a NaN in V.  Where some row does not see all of the chunk, tokens that no row sees are
        // cleared, and NaN codes of the others are taken out and given back to the rows that see them.
        bool nans = false;
        if (!whole) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int left = page[SUB == 1 ? 0 : u >> 1] >= 0 ? w.keys - token(u) : 0;     // (beyond the longest row lies at most the chunk's end)
                const uint32_t keep = tokens_left(left);
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    vw[i][u] &= keep;
                    nans = nans | (nan_bytes(vw[i][u], vs[SUB == 1 ? 0 : u >> 1]) != 0);
                }
            }
            nans = __any(nans);
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            uint32_t bad[4] = {0, 0, 0, 0};
            if (nans) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    bad[u] = nan_bytes(vw[i][u], vs[SUB == 1 ? 0 : u >> 1]);
                    vw[i][u] &= ~bad[u];
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const v8bf v = to_bf16(vw[i][2 * k], vw[i][2 * k + 1], vs[SUB == 1 ? 0 : k]);
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int j = PROBS - 1; j >= 0; --j) acc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[r][k][j], acc[r][i], 0, 0, 0);
            }
            if (nans) {
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    v4f hit{0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        v8bf sees;
#pragma unroll
                        for (int j = 0; j < 8; ++j) sees[j] = (__bf16)(token(2 * k + (j >> 2)) + (j & 3) < seen[r] ? 1.0f : 0.0f);
                        hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones_where(bad[2 * k], bad[2 * k + 1]), sees, hit, 0, 0, 0);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (hit[j] > 0.0f) acc[r][i][j] = NAN;
                }
            }
        }
    }

    // the four waves' sums: all of them into LDS before the first branch
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        l[r] += __shfl_xor(l[r], 16);
        l[r] += __shfl_xor(l[r], 32);
        if constexpr (PROBS == 1) {
            div[r] += __shfl_xor(div[r], 16);
            div[r] += __shfl_xor(div[r], 32);
        } else {
            div[r] = l[r];
        }
        s_sums[r][wave][n][0] = m[r];                                          // (the same from four lanes)
        s_sums[r][wave][n][1] = l[r];
        s_sums[r][wave][n][2] = div[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) top = fmaxf(top, s_sums[r][k][n][0]);
        // a wave without a number among its logits has m = -inf, and sums of 0, or NaN to pass on
        const float f = m[r] == -INFINITY ? (l[r] == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(m[r] - top);
#pragma unroll
        for (int i = 0; i < DT; ++i)
            *reinterpret_cast<float4*>(&s_o[r][wave][n][16 * i + 4 * h4]) = make_float4(acc[r][i][0] * f, acc[r][i][1] * f, acc[r][i][2] * f, acc[r][i][3] * f);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int rr = threadIdx.x >> 4, row = w.r0 + 16 * r + rr;
        if (row < w.rows) {
            float all = -INFINITY, total = 0.0f, divisor = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) all = fmaxf(all, s_sums[r][k][rr][0]);
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float mk = s_sums[r][k][rr][0], f = mk == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mk - all);
                total += s_sums[r][k][rr][1] * f;
                divisor += s_sums[r][k][rr][2] * f;
            }
            const bool last = w.active <= 1;
            const float inv = last ? 1.0f / (divisor == 0.0f ? 1.0f : divisor) : 1.0f;
            int tk, hd;
            row_at(places, 16 * r + rr, &tk, &hd);
            tk += w.begin;
            hd += head * a.group;
            const int64_t slot = ((int64_t)blockIdx.x * a.splits + z) * R + 16 * r + rr;
            constexpr int C = D / 16;                                          // channels of a thread
            float y[C];
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int ch = (threadIdx.x & 15) * C + j;
                y[j] = (s_o[r][0][rr][ch] + s_o[r][1][rr][ch] + s_o[r][2][rr][ch] + s_o[r][3][rr][ch]) * inv;
            }
            if (last) {
                char* at = a.o + (int64_t)tk * a.ot + (int64_t)hd * a.oh + (threadIdx.x & 15) * C * sizeof(T);
#pragma unroll
                for (int j = 0; j < C; ++j) Pack<T>::put(at + j * sizeof(T), y[j]);
                if (a.lse && (threadIdx.x & 15) == 0)
                    a.lse[(int64_t)hd * a.b.tokens + tk] = total == 0.0f ? -INFINITY : (all == -INFINITY ? 0.0f : all) * kLn2 + logf(total);
            } else {
#pragma unroll
                for (int j = 0; j < C; ++j) a.part_o[slot * D + (threadIdx.x & 15) * C + j] = y[j];
                if ((threadIdx.x & 15) == 0) a.part_sums[slot] = make_float4(all, total, divisor, 0.0f);
            }
        }
    }
}

// The pieces of a row, joined in their order, eight reads on their way at once: a wave per row, or for large tiles (whose place takes a search) four rows.
template <typename T, int D, int R, bool TILE>
__global__ __launch_bounds__(kThreads) void k_cache_attn_join(const Args a) {
    constexpr int C = D / 64, AHEAD = 8, EACH = TILE ? 4 : 1;
    const int items = a.workgroups / a.c.heads, at = a.whole + blockIdx.x, lane = threadIdx.x & 63;
    int head = at / items;
    Walk w;
    if (TILE ? !sorted_walk<R>(a, at, a.splits, &head, &w) : !tile_walk<R>(a, at % items, a.splits, &w)) return;
    if (w.active <= 1) return;
    for (int n = 0; n < EACH; ++n) {
        const int r = (kWaves * blockIdx.y + (threadIdx.x >> 6)) * EACH + n, row = w.r0 + r;
        if (row >= w.rows) return;
        const int64_t first = (int64_t)blockIdx.x * a.splits * R + r;              // pieces are R slots apart
        float m = -INFINITY, l = 0.0f, div = 0.0f;
        if (lane < w.active) {
            const float4 sums = a.part_sums[first + (int64_t)lane * R];
            m = sums.x;
            l = sums.y;
            div = sums.z;
        }
        float top = m;
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
        const float f = m == -INFINITY ? (l == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(m - top);
        float total = l * f, divisor = div * f;
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) {
            total += __shfl_xor(total, i);
            divisor += __shfl_xor(divisor, i);
        }
        float y[C];
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = 0.0f;
        for (int k0 = 0; k0 < w.active; k0 += AHEAD) {
            float x[AHEAD][C];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int j = 0; j < C; ++j) x[k][j] = a.part_o[(first + (int64_t)min(k0 + k, w.active - 1) * R) * D + lane * C + j];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const float g = __shfl(f, k0 + k);                                 // (0 behind the last: at most 64 pieces, in steps of 8)
#pragma unroll
                for (int j = 0; j < C; ++j) y[j] = fmaf(x[k][j], g, y[j]);
            }
        }
        const float inv = divisor == 0.0f ? 0.0f : 1.0f / divisor;
        const int tk = w.begin + row / a.group, hd = head * a.group + row % a.group;
        char* to = a.o + (int64_t)tk * a.ot + (int64_t)hd * a.oh + lane * C * sizeof(T);
#pragma unroll
        for (int j = 0; j < C; ++j) Pack<T>::put(to + j * sizeof(T), y[j] * inv);
        if (a.lse && lane == 0) a.lse[(int64_t)hd * a.b.tokens + tk] = total == 0.0f ? -INFINITY : (top == -INFINITY ? 0.0f : top) * kLn2 + logf(total);
    }
}

template <typename T, int D, int P, int NR>
void launch(const Args& a, hipStream_t st) {
    k_cache_attn_rows<T, D, P, NR><<<dim3((unsigned)a.workgroups, (unsigned)a.splits), kThreads, 0, st>>>(a);
    if (a.splits > 1) k_cache_attn_join<T, D, 16 * NR, false><<<dim3(a.workgroups, 4 * NR), kThreads, 0, st>>>(a);
}
template <typename T, int D, int P>
void launch_rows(const Args& a, int rows, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (rows == 32) return launch<T, D, P, 2>(a, st);
    }
    launch<T, D, P, 1>(a, st);
}
template <typename T, int D>
void launch_pages(const Args& a, int rows, hipStream_t st) {
    if (a.c.page_tokens == 128) launch_rows<T, D, 128>(a, rows, st);
    else if (a.c.page_tokens == 64) launch_rows<T, D, 64>(a, rows, st);
    else launch_rows<T, D, 32>(a, rows, st);
}

// The lanes of the wave that joins them.  Too few for a lone sequence of one or two cached heads: 264000 keys, 1 head 44 us, 1.6 TB/s; 4 heads 53 us.
constexpr int kMaxSplits = 64;

}  // namespace

CacheAttnPlan cache_attn_plan(const CacheArgs& c, const BatchArgs& b, bool bf16, int group, int cus) {
    CacheAttnPlan p{};
    const int64_t rows = (int64_t)b.tokens * group;
    // Rows of a sequence and cached head (128 channels; us with tiles of 256 and of 32): 16 heads of 16 sequences, 576 keys: 64 rows 29 and 45, 96 rows 34 and 69; 4
    // heads of 32 sequences, 2100 keys: 64 rows 67 and 51, 96 rows 68 and 79.  Fewer tiles than half the compute units have to be cut into more
    // pieces: 8 heads of 8 sequences, 4200 keys: 128 rows 83 and 77, 192 rows 86 and 106; 8 heads of one, 8400 keys: 192 rows 44 and 39, 256 rows 50 and 47.
    // The average decides for all sequences: a batch of prompts and single tokens has one of the two kernels for both.
    p.tile = bf16 && rows >= (2ll * b.sequences * c.heads >= cus ? 96 : 192) * b.sequences;
    // Tiles of 32 rows share a chunk's codes between two products: 64 rows 50 us, as 16 and 16 66 us; for a single one they only cost (5 rows: 74 us, 16 rows
    // a tile 68).  In fp32, with three parts to every operand, 16 rows are ahead (1500 rows over 4000 keys, 12 heads: 165 us, 32 rows a tile 247).
    p.rows = p.tile ? 256 : bf16 && rows > 16ll * b.sequences ? 32 : 16;
    p.workgroups = (rows / p.rows + b.sequences) * c.heads;
    const int64_t chunks = ((int64_t)b.max_pages * c.page_tokens + kChunk - 1) / kChunk;
    // Pieces of the rows kernel have two chunks a wave at least, or four where that leaves eight to a compute unit (48 ragged sequences of up to 16384 keys: 69 us,
    // with two 72; 8 sequences of 6144 keys and 15 rows each: two 20 us, with four 26, with one 26).  `chunks` goes by the width of the page table.
    const int64_t likely = std::max<int64_t>(b.sequences, (rows + p.rows - 1) / p.rows) * c.heads;      // tiles, unless the batch is very uneven
    p.least = p.tile ? 16 : likely * ((chunks + 4 * kWaves - 1) / (4 * kWaves)) >= 8ll * cus ? 4 * kWaves : 2 * kWaves;
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>((chunks + p.least - 1) / p.least, kMaxSplits));
    if (p.tile) {
        // One workgroup to a compute unit.  Rounds of tiles that fill them all stay whole; those of the last round are cut into the number of
        // pieces whose rounds take least, a piece costing some eight chunks by itself (its first chunk, its partial sums, joining them).
        p.whole = p.workgroups / cus * cus;
        if (p.whole % 8) p.whole = 0;        // (eight XCDs)
        const int64_t rest = p.workgroups - p.whole;
        double best = 1e300;
        p.splits = 1;
        for (int64_t s = 1; rest > 0 && s <= most; ++s) {
            const double time = (double)((rest * s + cus - 1) / cus) * ((double)chunks / s + (s > 1 ? 8 : 0));
            if (time < best * 0.99) { best = time; p.splits = (int)s; }
        }
        if (p.splits == 1) p.whole = 0;
    } else {
        // Twelve pieces to a compute unit, which holds two: with four the last ones keep those 48 sequences at 81 us instead of 69.
        p.splits = (int)std::min<int64_t>((12ll * cus + likely - 1) / likely, most);
    }
    p.scratch = p.splits > 1 ? (size_t)(p.workgroups - p.whole) * p.splits * p.rows * (c.d + 4) * sizeof(float) : 0;
    return p;
}

hipError_t launch_cache_attn(const CacheArgs& c, const BatchArgs& b, bool bf16, const void* Q, int64_t qt, int64_t qh, void* O, int64_t ot, int64_t oh,
                             float* lse, int group, bool causal, const CacheAttnPlan& p, void* scratch, hipStream_t st) {
    const int es = bf16 ? 2 : 4;
    Args a{};
    a.c = c;
    a.b = b;
    a.q = static_cast<const char*>(Q);
    a.o = static_cast<char*>(O);
    a.qt = qt * es; a.qh = qh * es; a.ot = ot * es; a.oh = oh * es;
    a.lse = lse;
    a.part_o = static_cast<float*>(scratch);
    a.part_sums = p.splits > 1 ? reinterpret_cast<float4*>(a.part_o + (size_t)(p.workgroups - p.whole) * p.splits * p.rows * c.d) : nullptr;
    a.group = group; a.causal = causal; a.splits = p.splits; a.least = p.least;
    a.workgroups = (int)p.workgroups;
    a.whole = (int)p.whole;
    a.scale = (float)(1.4426950408889634 / std::sqrt((double)c.d));
    if (p.tile) {
        launch_cache_attn_tile(a, st);
        if (p.splits > 1) {
            if (c.d == 128) k_cache_attn_join<__bf16, 128, 256, true><<<dim3(a.workgroups - a.whole, 256 / 16), kThreads, 0, st>>>(a);
            else k_cache_attn_join<__bf16, 64, 256, true><<<dim3(a.workgroups - a.whole, 256 / 16), kThreads, 0, st>>>(a);
        }
    } else if (bf16) {
        if (c.d == 128) launch_pages<__bf16, 128>(a, p.rows, st); else launch_pages<__bf16, 64>(a, p.rows, st);
    } else {
        if (c.d == 128) launch_pages<float, 128>(a, p.rows, st); else launch_pages<float, 64>(a, p.rows, st);
    }
    return hipGetLastError();
}

}  // namespace dr
