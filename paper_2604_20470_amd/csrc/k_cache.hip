// Appending keys and values to the paged e4m3 cache.  A workgroup owns one page of the keys or of the values, for a few heads one after the other: it
// reads the page's new tokens of a head once, rotates (keys), takes the largest magnitude, makes it the page's power of two, and writes codes,
// while the next head's tokens are on their way.  The angles are the same for all heads: their cosines and sines stay in registers.
// Nothing waits for another workgroup, and a page that already holds tokens is rescaled by the workgroup that adds to it.
// A power of two loses nothing against amax / 448 here: e4m3 is a floating format, its relative step does not depend on the scale,
// and growing the scale of codes that are there moves exponents only.
// Keys are rotated in 64 bits and rounded to fp32 once: an error of an fp32 rotation (1e-7) would turn one code in a million to its
// neighbour, 6 % away.
// Bound by memory: es + 1 bytes an element.  Values are held with tokens innermost (the second matrix product contracts over tokens),
// so the values' workgroup turns its tile around in LDS, four tokens to a word.  10800 tokens of 40 heads of 128 bf16 channels: 102 us, 3.2 TB/s, of which
// 41 us are the vector ALU's; 20 heads in fp32, half the elements, 54 us, 5.1 TB/s.
#include "stream_common.h"

namespace dr {
namespace {

using namespace stream;

constexpr int W = 4;                     // channels of a vector: 16 bytes of fp32, 8 of bf16
constexpr int kLeastExp = -100;          // of a scale: 2^-100 is far above the subnormals of bf16 and fp32, which the products would lose

struct AppendArgs {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    int32_t pages, heads;
    int32_t per;                         // heads of a workgroup
    BatchArgs b;
    const char *nk, *nv;                 // new keys, values
    int64_t kt, kh, vt, vh;              // bytes
    const int32_t* pos;                  // NULL: places in the sequence
    int64_t pos_axis;
    RopeTable r;
};

// cos and sin as rope_cos_sin's, in 64 bits: all bits of the fraction of a turn, two Taylor polynomials (truncated at 5e-17 and 1e-15).
__device__ __forceinline__ void cos_sin64(int32_t pos, uint64_t turn, double mscale, double& c, double& s) {
    const uint64_t t = (uint64_t)(int64_t)pos * turn + (1ull << 61);          // an eighth of a turn
    const uint32_t quarter = (uint32_t)(t >> 62);
    const double x = (double)((int64_t)(t & 0x3fffffffffffffffull) - (1ll << 61)) * (6.283185307179586476925 / 18446744073709551616.0), xx = x * x;
    double b = fma(xx, -1.0 / 1307674368000.0, 1.0 / 6227020800.0);
    b = fma(b, xx, -1.0 / 39916800.0);
    b = fma(b, xx, 1.0 / 362880.0);
    b = fma(b, xx, -1.0 / 5040.0);
    b = fma(b, xx, 1.0 / 120.0);
    b = fma(b, xx, -1.0 / 6.0);
    b = fma(b * xx, x, x) * mscale;
    double a = fma(xx, -1.0 / 87178291200.0, 1.0 / 479001600.0);
    a = fma(a, xx, -1.0 / 3628800.0);
    a = fma(a, xx, 1.0 / 40320.0);
    a = fma(a, xx, -1.0 / 720.0);
    a = fma(a, xx, 1.0 / 24.0);
    a = fma(a, xx, -0.5);
    a = fma(a, xx, 1.0) * mscale;
    c = (quarter & 1) ? b : a;                                               // |cos|, |sin|
    s = (quarter & 1) ? a : b;
    c = (quarter + 1) & 2 ? -c : c;
    s = quarter & 2 ? -s : s;
}

// The largest magnitude of a workgroup, infinity if there is one, NaN left out; `part` is another one in the next call.
template <int THREADS>
__device__ __forceinline__ float block_max(float x, float* part) {
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) x = fmaxf(x, __shfl_xor(x, i));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) x = fmaxf(x, part[i]);
    return x;
}
// Infinities saturate, whatever the scale: they count as the largest number does not.
__device__ __forceinline__ float finite(float x) { return fabsf(x) == INFINITY ? 0.0f : x; }

// Smallest e >= kLeastExp with amax <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int exponent_for(float amax) {
    return max((int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 127 - 8, kLeastExp);
}
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23 & 255u) - 127; }

// Four codes under a scale that has grown: 2^(old - new) of them, rounded again.
__device__ __forceinline__ uint32_t shrink(uint32_t w, float f) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return codes_of(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
}
__device__ __forceinline__ float shrink_factor(int old, int now) { return exp2_int(max(old - now, -126)); }

template <typename T>
__device__ __forceinline__ float key_channel(const AppendArgs& a, const char* row, int64_t token, int place, int c) {
    if (c >= a.r.dim) return Pack<T>::one(row + (int64_t)c * sizeof(T));
    const int half = a.r.dim / 2;
    const int pair = a.r.interleaved ? c >> 1 : (c < half ? c : c - half);
    const bool second = a.r.interleaved ? (c & 1) : c >= half;
    const int other = a.r.interleaved ? c ^ 1 : (second ? c - half : c + half);
    double co, si;
    cos_sin64(a.pos ? a.pos[rope_axis(a.r, pair) * a.pos_axis + token] : place, a.r.turn[pair], a.r.mscale, co, si);
    const double x = Pack<T>::one(row + (int64_t)c * sizeof(T)), z = Pack<T>::one(row + (int64_t)other * sizeof(T));
    return (float)fma(x, co, second ? z * si : -(z * si));
}

// Two halves of W channels, turned.  `apart`: q holds the other halves of p's pairs; else pairs lie side by side.
__device__ __forceinline__ void turn(bool apart, const double (&c)[W], const double (&s)[W], float (&p)[W], float (&q)[W]) {
    if (apart) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const double y = p[j], z = q[j];
            p[j] = (float)fma(y, c[j], -(z * s[j]));
            q[j] = (float)fma(z, c[j], y * s[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < W; j += 2) {
            const double y = p[j], z = p[j + 1], v = q[j], w = q[j + 1];
            p[j] = (float)fma(y, c[j / 2], -(z * s[j / 2]));
            p[j + 1] = (float)fma(z, c[j / 2], y * s[j / 2]);
            q[j] = (float)fma(v, c[W / 2 + j / 2], -(w * s[W / 2 + j / 2]));
            q[j + 1] = (float)fma(w, c[W / 2 + j / 2], v * s[W / 2 + j / 2]);
        }
    }
}
// Its angles; 0 for a unit that is copied, for which no position is read.
__device__ __forceinline__ void angles(const AppendArgs& a, int u, int64_t token, int place, double (&c)[W], double (&s)[W]) {
    const bool turned = unit_positions<W>(a.r.dim, a.r.end0, a.r.end1, u, [&](int axis) { return a.pos ? a.pos[axis * a.pos_axis + token] : place; },
                                          [&](int j, int pair, int pos) { cos_sin64(pos, a.r.turn[pair], a.r.mscale, c[j], s[j]); });
    if (turned) return;
#pragma unroll
    for (int j = 0; j < W; ++j) c[j] = s[j] = 0.0;
}
// Channels of unit u of a key: W from ca on and W from cb on.
__device__ __forceinline__ void channels(const AppendArgs& a, int u, bool& turned, int& ca, int& cb) {
    turned = 2 * W * u < a.r.dim;
    const bool apart = turned && !a.r.interleaved;
    ca = apart ? u * W : 2 * W * u;
    cb = apart ? a.r.dim / 2 + u * W : ca + W;
}
__device__ __forceinline__ float largest(const float (&x)[W], float most) {
#pragma unroll
    for (int j = 0; j < W; ++j) most = fmaxf(most, fabsf(x[j]));
    return most;
}
__device__ __forceinline__ float largest_finite(const float (&x)[W], float most) {
#pragma unroll
    for (int j = 0; j < W; ++j) most = fmaxf(most, fabsf(finite(x[j])));
    return most;
}
// Codes of W numbers under a scale of 1 / f, which keeps finite ones below the largest code.
__device__ __forceinline__ void put_codes(uint8_t* at, const float (&x)[W], float f, bool infinities) {
    float y[W];
#pragma unroll
    for (int k = 0; k < W; ++k) y[k] = infinities ? saturate(x[k] * f) : x[k] * f;
    *reinterpret_cast<uint32_t*>(at) = codes_of(y[0], y[1], y[2], y[3]);
}
// Where the page held tokens: its scale, and its codes if that grows.
__device__ __forceinline__ void regrow(uint8_t* page, int bytes, int old, int e, int threads) {
    uint32_t* words = reinterpret_cast<uint32_t*>(page);
    const float f = shrink_factor(old, e);
    for (int i = threadIdx.x; i < bytes / 4; i += threads) words[i] = shrink(words[i], f);
}
// The values' tile of codes, [channel][word of four slots], to its page.  Bytes of a word that are new: slots max(4 k, slot) ..
// min(4 k + 3, slot + m - 1); what lies behind them stays as it was.
template <int D, int P, int THREADS>
__device__ __forceinline__ void put_values(uint8_t* page, const uint32_t* tile, const Range& g, int old, int e) {
    constexpr int Q = P / 4, LD = Q + 1;
    const bool grown = g.slot && e > old;
    uint32_t* words = reinterpret_cast<uint32_t*>(page);
    if (g.m == P) {                            // a page that is new throughout
#pragma unroll 4
        for (int i = threadIdx.x; i < Q * D; i += THREADS) words[i] = tile[i / Q * LD + i % Q];
        return;
    }
    const int k0 = grown ? 0 : g.slot / 4, n = (g.slot + g.m + 3) / 4 - k0;
    const float f = shrink_factor(old, e);
    for (int i = threadIdx.x; i < n * D; i += THREADS) {
        const int c = i / n, k = k0 + (i - c * n);
        const uint32_t w = tile[c * LD + k];
        const int lo = max(g.slot - 4 * k, 0), hi = min(g.slot + g.m - 4 * k, 4);
        uint32_t* at = words + c * Q + k;
        if (lo == 0 && hi == 4) {
            *at = w;
        } else if (!grown) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t >= lo && t < hi) reinterpret_cast<uint8_t*>(at)[t] = (uint8_t)(w >> (8 * t));
        } else {
            const uint32_t there = *at, kept = shrink(there, f);
            const uint32_t from = lo >= 4 ? 0u : 0xffffffffu << (8 * lo), below = hi >= 4 ? 0xffffffffu : (1u << (8 * hi)) - 1u;
            *at = (w & from & below) | (kept & ~from) | (there & ~below);
        }
    }
}

// ---- Many tokens a page: a thread has two items of 2 W channels of a token, or one of W channels of four tokens; heads one after the other
template <int D, int P>
constexpr int kMany = P * D / 16;

template <typename T, int D, int P>
__device__ __forceinline__ void append_keys(const AppendArgs& a, const Range& g, float (&part)[3][16]) {
    constexpr int U = D / (2 * W), THREADS = kMany<D, P>, PER = P * U / THREADS;
    static_assert(PER * THREADS == P * U, "");
    const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.heads);
    Four<T> next[PER][2];
    auto load = [&](int h) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int id = i * THREADS + threadIdx.x;
            int ca, cb;
            bool turned;
            channels(a, id % U, turned, ca, cb);
            const char* r = a.nk + h * a.kh + (int64_t)(g.token + min(id / U, g.m - 1)) * a.kt;      // (rows behind the last: that one again)
            next[i][0].template get<true>(r + ca * (int)sizeof(T));
            next[i][1].template get<true>(r + cb * (int)sizeof(T));
        }
    };
    load(h0);
    double c[PER][W], s[PER][W];
    if (a.r.dim) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int id = i * THREADS + threadIdx.x, row = min(id / U, g.m - 1);
            angles(a, id % U, (int64_t)g.token + row, g.place + row, c[i], s[i]);
        }
    }
    for (int h = h0; h < h1; ++h) {
        float* scale = a.k_scale + (int64_t)g.page * a.heads + h;
        const int old = g.slot ? exponent_of(*scale) : kLeastExp;
        float p[PER][W], q[PER][W], most = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            next[i][0].values(p[i]);
            next[i][1].values(q[i]);
            if (a.r.dim) {
                float x[W], y[W];
#pragma unroll
                for (int j = 0; j < W; ++j) { x[j] = p[i][j]; y[j] = q[i][j]; }
                turn(!a.r.interleaved, c[i], s[i], x, y);
                const bool turned = 2 * W * ((i * THREADS + threadIdx.x) % U) < a.r.dim;
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    p[i][j] = turned ? x[j] : p[i][j];
                    q[i][j] = turned ? y[j] : q[i][j];
                }
            }
            most = largest(q[i], largest(p[i], most));
        }
        if (h + 1 < h1) load(h + 1);
        most = block_max<THREADS>(most, part[(h - h0) & 1]);
        const bool infinities = most == INFINITY;
        if (infinities) {
            most = 0.0f;
#pragma unroll
            for (int i = 0; i < PER; ++i) most = largest_finite(q[i], largest_finite(p[i], most));
            most = block_max<THREADS>(most, part[2]);
        }
        const int e = max(exponent_for(most), old);
        uint8_t* page = a.k + ((int64_t)g.page * a.heads + h) * (P * D);
        const float f = exp2_int(-e);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int id = i * THREADS + threadIdx.x;
            int ca, cb;
            bool turned;
            channels(a, id % U, turned, ca, cb);
            if (id / U < g.m) {
                put_codes(page + (g.slot + id / U) * D + ca, p[i], f, infinities);
                put_codes(page + (g.slot + id / U) * D + cb, q[i], f, infinities);
            }
        }
        if (g.slot && e > old) regrow(page, g.slot * D, old, e, THREADS);
        if (threadIdx.x == 0) *scale = exp2_int(e);      // (all have read the old one: the workgroup's maximum lies between)
    }
}

template <typename T, int D, int P>
__device__ __forceinline__ void append_values(const AppendArgs& a, const Range& g, uint32_t* tile, float (&part)[3][16]) {
    constexpr int U = D / 4, LD = P / 4 + 1, THREADS = kMany<D, P>;
    const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.heads), k = threadIdx.x / U, u = threadIdx.x % U;
    Four<T> next[4];
    auto load = [&](int h) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = 4 * k + t - g.slot;                                // (rows that are not there: zeros)
            next[t].template get<true>(a.nv + h * a.vh + (int64_t)(g.token + min(max(row, 0), g.m - 1)) * a.vt + u * (4 * (int)sizeof(T)));
            next[t].keep(row >= 0 && row < g.m);
        }
    };
    load(h0);
    for (int h = h0; h < h1; ++h) {
        float* scale = a.v_scale + (int64_t)g.page * a.heads + h;
        const int old = g.slot ? exponent_of(*scale) : kLeastExp;
        float x[4][4], most = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            next[t].values(x[t]);
            most = largest(x[t], most);
        }
        if (h + 1 < h1) load(h + 1);
        most = block_max<THREADS>(most, part[(h - h0) & 1]);
        const bool infinities = most == INFINITY;
        if (infinities) {
            most = 0.0f;
#pragma unroll
            for (int t = 0; t < 4; ++t) most = largest_finite(x[t], most);
            most = block_max<THREADS>(most, part[2]);
        }
        const int e = max(exponent_for(most), old);
        const float f = exp2_int(-e);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[t][j] *= f;
        if (infinities) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[t][j] = saturate(x[t][j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) tile[(u * 4 + j) * LD + k] = codes_of(x[0][j], x[1][j], x[2][j], x[3][j]);
        __syncthreads();
        put_values<D, P, THREADS>(a.v + ((int64_t)g.page * a.heads + h) * (P * D), tile, g, old, e);
        if (threadIdx.x == 0) *scale = exp2_int(e);
    }
}

template <typename T, int D, int P>
__global__ __launch_bounds__((kMany<D, P>)) void k_cache_append_many(const AppendArgs a) {
    __shared__ uint32_t tile[D * (P / 4 + 1)];
    __shared__ float part[3][16];
    const Range g = range_of(a.b, a.pages, P, find_place(a.b, blockIdx.x, 1, P, 2));
    if (g.m <= 0) return;
    if (blockIdx.z == 0) append_keys<T, D, P>(a, g, part);
    else append_values<T, D, P>(a, g, tile, part);
}

// ---- Few tokens a page, or rows that do not come in vectors: nothing is kept, the tokens are read (from the cache) and turned twice
constexpr int kFew = 256;

template <typename T, int D, int P, bool VEC>
__global__ __launch_bounds__(kFew) void k_cache_append_few(const AppendArgs a) {
    constexpr int U = D / (2 * W), UV = D / 4, LD = P / 4 + 1;
    __shared__ uint32_t tile[D * LD];
    __shared__ float part[kFew / 64];
    const Range g = range_of(a.b, a.pages, P, find_place(a.b, blockIdx.x, 1, P, 2));
    if (g.m <= 0) return;
    const int h = blockIdx.y;
    const bool keys = blockIdx.z == 0;
    float* scale = (keys ? a.k_scale : a.v_scale) + (int64_t)g.page * a.heads + h;
    const int old = g.slot ? exponent_of(*scale) : kLeastExp;
    auto key = [&](int id, float (&p)[W], float (&q)[W], int& ca, int& cb) {
        const int row = id / U, u = id % U;
        const char* r = a.nk + h * a.kh + (int64_t)(g.token + row) * a.kt;
        if constexpr (VEC) {
            bool turned;
            channels(a, u, turned, ca, cb);
            Four<T> v, w;
            v.template get<true>(r + ca * (int)sizeof(T));
            w.template get<true>(r + cb * (int)sizeof(T));
            v.values(p);
            w.values(q);
            if (turned) {
                double c[W], s[W];
                angles(a, u, (int64_t)g.token + row, g.place + row, c, s);
                turn(!a.r.interleaved, c, s, p, q);
            }
        } else {
            ca = 2 * W * u;
            cb = ca + W;
#pragma unroll
            for (int j = 0; j < W; ++j) {
                p[j] = key_channel<T>(a, r, (int64_t)g.token + row, g.place + row, ca + j);
                q[j] = key_channel<T>(a, r, (int64_t)g.token + row, g.place + row, cb + j);
            }
        }
    };
    // values: words first .. of four slots
    const int first = g.slot / 4, words = (g.slot + g.m + 3) / 4 - first, items = keys ? g.m * U : words * UV;
    auto value = [&](int id, float (&x)[4][4]) {
        const int k = first + id / UV, u = id % UV;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = 4 * k + t - g.slot;
            Four<T> v;
            v.template get<VEC>(a.nv + h * a.vh + (int64_t)(g.token + min(max(row, 0), g.m - 1)) * a.vt + u * (4 * (int)sizeof(T)));
            v.keep(row >= 0 && row < g.m);
            v.values(x[t]);
        }
    };
    float most = 0.0f;
    for (int id = threadIdx.x; id < items; id += kFew) {
        if (keys) {
            float p[W], q[W];
            int ca, cb;
            key(id, p, q, ca, cb);
            most = largest_finite(q, largest_finite(p, most));
        } else {
            float x[4][4];
            value(id, x);
#pragma unroll
            for (int t = 0; t < 4; ++t) most = largest_finite(x[t], most);
        }
    }
    const int e = max(exponent_for(block_max<kFew>(most, part)), old);
    const float f = exp2_int(-e);
    for (int id = threadIdx.x; id < items; id += kFew) {
        if (keys) {
            float p[W], q[W];
            int ca, cb;
            key(id, p, q, ca, cb);
            uint8_t* at = a.k + ((int64_t)g.page * a.heads + h) * (P * D) + (g.slot + id / U) * D;
            put_codes(at + ca, p, f, true);
            put_codes(at + cb, q, f, true);
        } else {
            float x[4][4];
            value(id, x);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                tile[(id % UV * 4 + j) * LD + first + id / UV] = codes_of(saturate(x[0][j] * f), saturate(x[1][j] * f), saturate(x[2][j] * f), saturate(x[3][j] * f));
        }
    }
    if (keys) {
        if (g.slot && e > old) regrow(a.k + ((int64_t)g.page * a.heads + h) * (P * D), g.slot * D, old, e, kFew);
    } else {
        __syncthreads();
        put_values<D, P, kFew>(a.v + ((int64_t)g.page * a.heads + h) * (P * D), tile, g, old, e);
    }
    if (threadIdx.x == 0) *scale = exp2_int(e);
}

template <typename T, int D, int P>
void launch(bool vec, bool few, const dim3& grid, const AppendArgs& a, hipStream_t st) {
    if (!vec) k_cache_append_few<T, D, P, false><<<grid, kFew, 0, st>>>(a);
    else if (few) k_cache_append_few<T, D, P, true><<<grid, kFew, 0, st>>>(a);
    else k_cache_append_many<T, D, P><<<grid, kMany<D, P>, 0, st>>>(a);
}
template <typename T, int D>
void launch_pages(int P, bool vec, bool few, const dim3& grid, const AppendArgs& a, hipStream_t st) {
    if (P == 128) launch<T, D, 128>(vec, few, grid, a, st);
    else if (P == 64) launch<T, D, 64>(vec, few, grid, a, st);
    else launch<T, D, 32>(vec, few, grid, a, st);
}

}  // namespace

hipError_t launch_cache_append(const CacheArgs& c, const BatchArgs& b, bool bf16, const void* K, const void* V, int64_t kt, int64_t kh, int64_t vt,
                               int64_t vh, const RopeTable& r, const int32_t* pos, int64_t pos_axis, int cus, hipStream_t st) {
    const int es = bf16 ? 2 : 4;
    AppendArgs a{};
    a.k = c.k; a.v = c.v; a.k_scale = c.k_scale; a.v_scale = c.v_scale; a.pages = c.pages; a.heads = c.heads;
    a.b = b;
    a.nk = static_cast<const char*>(K); a.nv = static_cast<const char*>(V);
    a.kt = kt * es; a.kh = kh * es; a.vt = vt * es; a.vh = vh * es;
    a.pos = pos; a.pos_axis = pos_axis;
    a.r = r;
    const auto odd = reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) | (uintptr_t)a.kt | (uintptr_t)a.kh | (uintptr_t)a.vt | (uintptr_t)a.vh;
    const bool vec = odd % (W * es) == 0 && r.dim % (2 * W) == 0;      // rows and pairs come in vectors
    // A workgroup of 4 waves that keeps nothing is ahead as long as it has few of a page's tokens; the other one has P d / 16 threads, so the limit goes by
    // that.  New tokens a sequence, us of this one and of the other, d = 128: 48 sequences, 8 heads, pages of 128: 1 token 7.7 and 21.7, 16 11.3 and 22.9, 48
    // 18.5 and 24.6, 64 20.7 and 21.5, 96 31.3 and 24.0; 8 sequences of 40 heads: 48 16.4 and 22.9, 64 21.6 and 17.4; one sequence: 32 7.0 and 8.0, 48 8.7 and
    // 8.2; 4 sequences, fp32, pages of 64: 16 5.8 and 6.3, 24 7.1 and 6.4, 64 10.4 and 6.4.  d = 64, pages of 64: 4 6.2 and 7.1, 16 7.7 and 7.3; pages of 32, fp32: 4 6.2
    // and 6.5, 16 6.6 and 6.4, 48 7.6 and 6.6.
    const bool few = !vec || b.tokens <= 3ll * c.page_tokens * c.d / 1024 * b.sequences;
    // Heads of a workgroup: as many as leave one round of waves (16 to a compute unit), eight at most.  10800 tokens of 40 heads of 128 channels: 8
    // heads 100 us, 4 heads 103, 2 heads 123, 1 head (its angles computed for each) 168; 9 sequences of 12 heads of 64: 2 heads 11.2 us, 1 and 4 13.4 and 13.7.
    const int64_t places = (int64_t)b.tokens / c.page_tokens + 2ll * b.sequences;
    const int64_t waves = 2 * places * c.heads * (c.page_tokens * c.d / 16 / 64), round = 16ll * cus;
    a.per = few ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(8, (waves + round / 2) / round));
    const dim3 grid((unsigned)places, (unsigned)((c.heads + a.per - 1) / a.per), 2u);
    if (bf16) { if (c.d == 128) launch_pages<__bf16, 128>(c.page_tokens, vec, few, grid, a, st); else launch_pages<__bf16, 64>(c.page_tokens, vec, few, grid, a, st); }
    else { if (c.d == 128) launch_pages<float, 128>(c.page_tokens, vec, few, grid, a, st); else launch_pages<float, 64>(c.page_tokens, vec, few, grid, a, st); }
    return hipGetLastError();
}

}  // namespace dr
