// Appending keys and values to the paged e4m3 cache.  One workgroup owns one (page, head) of the keys or of the values: it reads the
// page's new tokens once, rotates (keys) in fp32, takes the largest magnitude, makes it the page's power of two, and writes codes.
// Nothing waits for another workgroup, and a page that already holds tokens is rescaled by the workgroup that adds to it.
// A power of two loses nothing against amax / 448 here: e4m3 is a floating format, its relative step does not depend on the scale,
// and growing the scale of codes that are there moves exponents only.
// Bound by memory: es + 1 bytes an element.  Values are held with tokens innermost (the second matrix product contracts over tokens),
// so the values' workgroup turns its tile around in LDS, four tokens to a word.
#include "stream_common.h"

namespace dr {
namespace {

using namespace stream;

constexpr int kThreads = 256;
constexpr int kLeastExp = -100;          // of a scale: 2^-100 is far above the subnormals of bf16 and fp32, which the products would lose

struct AppendArgs {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    int32_t pages, heads;
    BatchArgs b;
    const char *nk, *nv;                 // new keys, values
    int64_t kt, kh, vt, vh;              // bytes
    const int32_t* pos;                  // NULL: places in the sequence
    int64_t pos_axis;
    int32_t vec;                         // rows and pairs come in 16-byte vectors
    RopeTable r;
};

__device__ __forceinline__ float block_max(float x) {
    __shared__ float part[kThreads / 64];
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) x = fmaxf(x, __shfl_xor(x, i));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}
// Magnitude that counts for the scale: infinities saturate and NaN stays whatever the scale is.
__device__ __forceinline__ float magnitude(float x) { const float y = fabsf(x); return y <= 3.402823466e38f ? y : 0.0f; }

// Smallest e >= kLeastExp with amax <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int exponent_for(float amax) {
    return max((int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 127 - 8, kLeastExp);
}
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23 & 255u) - 127; }

// Four codes under a scale that has grown: 2^(old - new) of them, rounded again.
__device__ __forceinline__ uint32_t shrink(uint32_t w, float f) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return to_e4m3<true>(b[0] * f, b[1] * f, to_e4m3<false>(a[0] * f, a[1] * f, 0));
}
__device__ __forceinline__ float shrink_factor(int old, int now) { return exp2_int(max(old - now, -126)); }

template <typename T>
__device__ __forceinline__ float key_channel(const AppendArgs& a, const char* row, int64_t token, int place, int c) {
    if (c >= a.r.dim) return Pack<T>::one(row + (int64_t)c * sizeof(T));
    const int half = a.r.dim / 2;
    const int pair = a.r.interleaved ? c >> 1 : (c < half ? c : c - half);
    const bool second = a.r.interleaved ? (c & 1) : c >= half;
    const int other = a.r.interleaved ? c ^ 1 : (second ? c - half : c + half);
    const int pos = a.pos ? a.pos[rope_axis(a.r, pair) * a.pos_axis + token] : place;
    const float2 cs = rope_cos_sin(pos, a.r.turn[pair]);
    const float x = Pack<T>::one(row + (int64_t)c * sizeof(T)), z = Pack<T>::one(row + (int64_t)other * sizeof(T));
    return a.r.mscale * cs.x * x + (second ? a.r.mscale * cs.y * z : -(a.r.mscale * cs.y * z));
}

template <typename T, int D, int P>
__device__ __forceinline__ void append_keys(const AppendArgs& a, const Range& g) {
    constexpr int W = Pack<T>::W, U = D / (2 * W), PER = (P * U + kThreads - 1) / kThreads;
    const int h = blockIdx.y;
    const char* base = a.nk + (int64_t)g.token * a.kt + h * a.kh;
    float x[PER][2 * W];
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int id = i * kThreads + threadIdx.x, row = id / U, u = id % U;
        if (row >= g.m) continue;
        const char* r = base + row * a.kt;
        const bool turned = 2 * W * u < a.r.dim, apart = turned && !a.r.interleaved;
        const int ca = a.vec && apart ? u * W : 2 * W * u, cb = a.vec && apart ? a.r.dim / 2 + u * W : ca + W;
        if (a.vec) {
            float p[W], q[W];
            Pack<T>::load(r + ca * (int)sizeof(T), p);
            Pack<T>::load(r + cb * (int)sizeof(T), q);
            if (turned) {
                float c[W], s[W];
                int axis = -1, pos = 0;
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const int k = rope_axis(a.r, u * W + j);
                    if (k != axis) pos = a.pos ? a.pos[k * a.pos_axis + g.token + row] : g.place + row;
                    axis = k;
                    const float2 cs = rope_cos_sin(pos, a.r.turn[u * W + j]);
                    c[j] = cs.x * a.r.mscale;
                    s[j] = cs.y * a.r.mscale;
                }
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    if (apart) {
                        x[i][j] = p[j] * c[j] - q[j] * s[j];
                        x[i][W + j] = q[j] * c[j] + p[j] * s[j];
                    } else {
                        const int k = j & ~1, m = j / 2;
                        x[i][j] = fmaf(p[j], c[m], (j & 1) ? p[k] * s[m] : -(p[k + 1] * s[m]));
                        x[i][W + j] = fmaf(q[j], c[W / 2 + m], (j & 1) ? q[k] * s[W / 2 + m] : -(q[k + 1] * s[W / 2 + m]));
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < W; ++j) { x[i][j] = p[j]; x[i][W + j] = q[j]; }
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < 2 * W; ++j) {
                const float y = key_channel<T>(a, r, (int64_t)g.token + row, g.place + row, ca + j);
#pragma unroll
                for (int k = 0; k < 2 * W; ++k) if (k == j) x[i][k] = y;      // (registers are not indexed at run time)
            }
        }
#pragma unroll
        for (int j = 0; j < 2 * W; ++j) amax = fmaxf(amax, magnitude(x[i][j]));
    }
    float* scale = a.k_scale + (int64_t)g.page * a.heads + h;
    const int old = g.slot ? exponent_of(*scale) : kLeastExp;
    const int e = max(exponent_for(block_max(amax)), old);
    uint8_t* page = a.k + ((int64_t)g.page * a.heads + h) * (P * D);
    const float f = exp2_int(-e);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int id = i * kThreads + threadIdx.x, row = id / U, u = id % U;
        if (row >= g.m) continue;
        const bool apart = a.vec && 2 * W * u < a.r.dim && !a.r.interleaved;
        const int ca = apart ? u * W : 2 * W * u, cb = apart ? a.r.dim / 2 + u * W : ca + W;
        uint32_t w[2 * W / 4];
#pragma unroll
        for (int j = 0; j < 2 * W / 4; ++j)
            w[j] = to_e4m3<true>(x[i][4 * j + 2] * f, x[i][4 * j + 3] * f, to_e4m3<false>(x[i][4 * j] * f, x[i][4 * j + 1] * f, 0));
        uint8_t* at = page + (g.slot + row) * D;
        if constexpr (W == 8) {
            *reinterpret_cast<uint2*>(at + ca) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2*>(at + cb) = make_uint2(w[2], w[3]);
        } else {
            *reinterpret_cast<uint32_t*>(at + ca) = w[0];
            *reinterpret_cast<uint32_t*>(at + cb) = w[1];
        }
    }
    if (g.slot && e > old) {
        uint32_t* words = reinterpret_cast<uint32_t*>(page);
        const float s = shrink_factor(old, e);
        for (int i = threadIdx.x; i < g.slot * D / 4; i += kThreads) words[i] = shrink(words[i], s);
    }
    if (threadIdx.x == 0) *scale = exp2_int(e);
}

// Values: thread items are four slots (a word of the page) by W channels.
template <typename T, int D, int P>
__device__ __forceinline__ void append_values(const AppendArgs& a, const Range& g, uint32_t* tile) {
    constexpr int W = Pack<T>::W, U = D / W, Q = P / 4, PER = (Q * U + kThreads - 1) / kThreads, LD = Q + 1;
    const int h = blockIdx.y;
    const char* base = a.nv + (int64_t)g.token * a.vt + h * a.vh;
    float x[PER][4][W];
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int id = i * kThreads + threadIdx.x, q = id / U, u = id % U;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = 4 * q + t - g.slot;
            const char* r = base + row * a.vt + (int64_t)u * (W * sizeof(T));
            if (row < 0 || row >= g.m) {
#pragma unroll
                for (int j = 0; j < W; ++j) x[i][t][j] = 0.0f;
            } else if (a.vec) {
                Pack<T>::load(r, x[i][t]);
            } else {
#pragma unroll
                for (int j = 0; j < W; ++j) x[i][t][j] = Pack<T>::one(r + j * (int)sizeof(T));
            }
#pragma unroll
            for (int j = 0; j < W; ++j) amax = fmaxf(amax, magnitude(x[i][t][j]));
        }
    }
    float* scale = a.v_scale + (int64_t)g.page * a.heads + h;
    const int old = g.slot ? exponent_of(*scale) : kLeastExp;
    const int e = max(exponent_for(block_max(amax)), old);
    const float f = exp2_int(-e);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int id = i * kThreads + threadIdx.x, q = id / U, u = id % U;
        if (q >= Q) continue;
#pragma unroll
        for (int j = 0; j < W; ++j)
            tile[(u * W + j) * LD + q] = to_e4m3<true>(x[i][2][j] * f, x[i][3][j] * f, to_e4m3<false>(x[i][0][j] * f, x[i][1][j] * f, 0));
    }
    __syncthreads();
    const bool grown = g.slot && e > old;
    const float s = shrink_factor(old, e);
    const int q0 = grown ? 0 : g.slot / 4, q1 = (g.slot + g.m + 3) / 4, nq = q1 - q0;
    uint32_t* words = reinterpret_cast<uint32_t*>(a.v + ((int64_t)g.page * a.heads + h) * (P * D));
    for (int i = threadIdx.x; i < nq * D; i += kThreads) {
        const int c = i / nq, q = q0 + (i - c * nq);
        uint32_t w = tile[c * LD + q];
        // bytes of the word that are new: slots max(4 q, slot) .. min(4 q + 3, slot + m - 1)
        const int lo = max(g.slot - 4 * q, 0), hi = min(g.slot + g.m - 4 * q, 4);
        if (lo > 0 || hi < 4) {
            const uint32_t there = words[c * Q + q], kept = grown ? shrink(there, s) : there;
            const uint32_t from = lo >= 4 ? 0u : 0xffffffffu << (8 * lo), below = hi >= 4 ? 0xffffffffu : (1u << (8 * hi)) - 1u;
            // earlier tokens, new ones, and what lies behind them as it was
            w = (w & from & below) | (kept & ~from) | (there & ~below);
        }
        words[c * Q + q] = w;
    }
    if (threadIdx.x == 0) *scale = exp2_int(e);
}

template <typename T, int D, int P>
__global__ __launch_bounds__(kThreads) void k_cache_append(const AppendArgs a) {
    __shared__ uint32_t tile[D * (P / 4 + 1)];
    const Range g = range_of(a.b, a.pages, P, find_place(a.b, blockIdx.x, 1, P, 2));
    if (g.m <= 0) return;
    if (blockIdx.z == 0) append_keys<T, D, P>(a, g);
    else append_values<T, D, P>(a, g, tile);
}

template <typename T, int D>
void launch_pages(int P, const dim3& grid, const AppendArgs& a, hipStream_t st) {
    if (P == 128) k_cache_append<T, D, 128><<<grid, kThreads, 0, st>>>(a);
    else if (P == 64) k_cache_append<T, D, 64><<<grid, kThreads, 0, st>>>(a);
    else k_cache_append<T, D, 32><<<grid, kThreads, 0, st>>>(a);
}

}  // namespace

hipError_t launch_cache_append(const CacheArgs& c, const BatchArgs& b, bool bf16, const void* K, const void* V, int64_t kt, int64_t kh, int64_t vt,
                               int64_t vh, const RopeTable& r, const int32_t* pos, int64_t pos_axis, hipStream_t st) {
    const int es = bf16 ? 2 : 4, W = 16 / es;
    AppendArgs a{};
    a.k = c.k; a.v = c.v; a.k_scale = c.k_scale; a.v_scale = c.v_scale; a.pages = c.pages; a.heads = c.heads;
    a.b = b;
    a.nk = static_cast<const char*>(K); a.nv = static_cast<const char*>(V);
    a.kt = kt * es; a.kh = kh * es; a.vt = vt * es; a.vh = vh * es;
    a.pos = pos; a.pos_axis = pos_axis;
    a.r = r;
    const auto odd = reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) | (uintptr_t)a.kt | (uintptr_t)a.kh | (uintptr_t)a.vt | (uintptr_t)a.vh;
    a.vec = odd % 16 == 0 && r.dim % (2 * W) == 0;
    const dim3 grid((unsigned)(b.tokens / c.page_tokens + 2 * b.sequences), (unsigned)c.heads, 2u);
    if (bf16) { if (c.d == 128) launch_pages<__bf16, 128>(c.page_tokens, grid, a, st); else launch_pages<__bf16, 64>(c.page_tokens, grid, a, st); }
    else { if (c.d == 128) launch_pages<float, 128>(c.page_tokens, grid, a, st); else launch_pages<float, 64>(c.page_tokens, grid, a, st); }
    return hipGetLastError();
}

}  // namespace dr
