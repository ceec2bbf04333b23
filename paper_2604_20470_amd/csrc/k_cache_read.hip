// Keys and values of cached tokens as dense rows: the inverse of the append.
//
// value = code * 2^e is exact in bf16 and in fp32.  A workgroup has the wanted tokens of one page, of the keys or of the values, for a few heads.  Keys lie as they are wanted: a lane makes
// 16 bytes of a token's row.  Values have their tokens innermost: a lane reads 16 tokens of as many channels, turns 4 x 4 bytes around with byte permutes in registers, and has 16 bytes of
// 16 rows to store; the lanes side by side store whole rows.  No LDS.
// Bound by memory: 1 + es bytes an element.  75600 tokens of 40 heads of 128 in bf16: 445 us, 5.2 TB/s.
#include "stream_common.h"

namespace dr {
namespace {

using namespace stream;

constexpr int kThreads = 256, kHeads = 4;       // heads of a workgroup

struct ReadArgs {
    CacheArgs c;
    BatchArgs b;
    char *k, *v;                                // NULL: not wanted
    int64_t kt, kh, vt, vh;                     // bytes
};

// Codes to 16 bytes of a row: eight channels of bf16, four of fp32.
template <typename T> struct Codes;
template <> struct Codes<__bf16> { uint32_t w[2]; };
template <> struct Codes<float> { uint32_t w[1]; };
template <typename T, bool VEC>
__device__ __forceinline__ void put_codes(char* at, const Codes<T>& c, float scale) {
    if constexpr (sizeof(T) == 2) {
        const v2bf p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[0], scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[0], scale, true),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[1], scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[1], scale, true)};
        if constexpr (VEC) {
            *reinterpret_cast<uint4*>(at) = make_uint4(__builtin_bit_cast(uint32_t, p[0]), __builtin_bit_cast(uint32_t, p[1]), __builtin_bit_cast(uint32_t, p[2]),
                                                       __builtin_bit_cast(uint32_t, p[3]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) reinterpret_cast<__bf16*>(at)[j] = p[j / 2][j & 1];
        }
    } else {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[0], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[0], true);
        const float x[4] = {a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale};
        if constexpr (VEC) {
            *reinterpret_cast<float4*>(at) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) reinterpret_cast<float*>(at)[j] = x[j];
        }
    }
}
// Bytes i of four words as one word, i = 0 .. 3.
__device__ __forceinline__ void turn_bytes(const uint32_t (&w)[4], uint32_t (&t)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);      // bytes 0, 0', 1, 1'
    const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);      // bytes 2, 2', 3, 3'
    t[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    t[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    t[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
    t[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}
// A page's scale: the power of two at or below it.
__device__ __forceinline__ float page_power(const float* scales, int64_t at) { return __uint_as_float(__float_as_uint(scales[at]) & 0x7f800000u); }

template <typename T, int D, int P, bool VEC>
__global__ __launch_bounds__(kThreads) void k_cache_read(const ReadArgs a) {
    constexpr int W = 16 / sizeof(T), C = D / W;  // channels of a lane; groups of them in a row
    const bool values = blockIdx.z != 0;
    char* to = values ? a.v : a.k;
    if (!to) return;
    const int64_t ts = values ? a.vt : a.kt, hs = values ? a.vh : a.kh;
    const Range g = read_range_of(a.b, a.c.pages, P, find_place(a.b, blockIdx.x, 1, P, 2));
    if (g.m == 0) return;
    const int head0 = blockIdx.y * kHeads, heads = min(kHeads, a.c.heads - head0);
    to += (int64_t)g.token * ts;                // row of the range's first token
    if (g.page < 0) {                           // nothing is stored for these tokens
        for (int i = threadIdx.x; i < heads * g.m * C; i += kThreads) {
            const int c = i % C, t = i / C % g.m, h = head0 + i / C / g.m;
            put_codes<T, VEC>(to + t * ts + h * hs + c * 16, Codes<T>{}, 1.0f);
        }
        return;
    }
    const int64_t page0 = (int64_t)g.page * a.c.heads + head0;
    if (!values) {
        constexpr int AHEAD = 4;
        const int n = heads * g.m * C;
        for (int i0 = threadIdx.x; i0 < n; i0 += AHEAD * kThreads) {
            Codes<T> w[AHEAD];
            float f[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int i = min(i0 + j * kThreads, n - 1), h = i / C / g.m, t = i / C - h * g.m;
                w[j] = *reinterpret_cast<const Codes<T>*>(a.c.k + (page0 + h) * (P * D) + (g.slot + t) * D + i % C * W);
                f[j] = page_power(a.c.k_scale, page0 + h);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int i = i0 + j * kThreads, h = i / C / g.m, t = i / C - h * g.m;
                if (i < n) put_codes<T, VEC>(to + t * ts + (head0 + h) * hs + i % C * 16, w[j], f[j]);
            }
        }
        return;
    }
    constexpr int GROUPS = P / 16;
    for (int i = threadIdx.x; i < heads * GROUPS * C; i += kThreads) {
        const int c = i % C, first = 16 * (i / C % GROUPS), h = i / C / GROUPS;
        if (first + 16 <= g.slot || first >= g.slot + g.m) continue;
        uint4 w[W];
        const uint8_t* at = a.c.v + (page0 + h) * (P * D) + c * W * P + first;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = *reinterpret_cast<const uint4*>(at + j * P);
        const float f = page_power(a.c.v_scale, page0 + h);
        char* row = to + (head0 + h) * hs + (first - g.slot) * ts + c * 16;
#pragma unroll
        for (int q = 0; q < 4; ++q) {           // four tokens
            uint32_t turned[W / 4][4];
            auto word = [&](int j) { return q == 0 ? w[j].x : q == 1 ? w[j].y : q == 2 ? w[j].z : w[j].w; };
#pragma unroll
            for (int j = 0; j < W / 4; ++j) {
                const uint32_t x[4] = {word(4 * j), word(4 * j + 1), word(4 * j + 2), word(4 * j + 3)};
                turn_bytes(x, turned[j]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = first + 4 * q + k;
                Codes<T> x;
#pragma unroll
                for (int j = 0; j < W / 4; ++j) x.w[j] = turned[j][k];
                if (t >= g.slot && t < g.slot + g.m) put_codes<T, VEC>(row + (4 * q + k) * ts, x, f);
            }
        }
    }
}

template <typename T, int D, int P>
void launch(const ReadArgs& a, bool wide, dim3 grid, hipStream_t st) {
    if (wide) k_cache_read<T, D, P, true><<<grid, kThreads, 0, st>>>(a);
    else k_cache_read<T, D, P, false><<<grid, kThreads, 0, st>>>(a);
}
template <typename T, int D>
void launch_pages(const ReadArgs& a, bool wide, dim3 grid, hipStream_t st) {
    if (a.c.page_tokens == 128) launch<T, D, 128>(a, wide, grid, st);
    else if (a.c.page_tokens == 64) launch<T, D, 64>(a, wide, grid, st);
    else launch<T, D, 32>(a, wide, grid, st);
}

}  // namespace

hipError_t launch_cache_read(const CacheArgs& c, const BatchArgs& b, bool bf16, void* K, void* V, int64_t kt, int64_t kh, int64_t vt, int64_t vh, bool wide, hipStream_t st) {
    const int es = bf16 ? 2 : 4;
    const ReadArgs a{c, b, static_cast<char*>(K), static_cast<char*>(V), kt * es, kh * es, vt * es, vh * es};
    const dim3 grid((unsigned)(b.tokens / c.page_tokens + 2 * b.sequences), (unsigned)((c.heads + kHeads - 1) / kHeads), 2);
    if (bf16) {
        if (c.d == 128) launch_pages<__bf16, 128>(a, wide, grid, st); else launch_pages<__bf16, 64>(a, wide, grid, st);
    } else {
        if (c.d == 128) launch_pages<float, 128>(a, wide, grid, st); else launch_pages<float, 64>(a, wide, grid, st);
    }
    return hipGetLastError();
}

}  // namespace dr
