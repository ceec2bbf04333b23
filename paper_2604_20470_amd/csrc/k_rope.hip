// Rotary positions over [B, H, N, d]: y0 = m (x0 cos - x1 sin), y1 = m (x1 cos + x0 sin) for every pair of channels; the gradient is the
// same with the sine's sign turned.  Bound by memory: every element is read once and written once, three operations each.  The
// cosines and sines (some 25 instructions a pair) depend on the token and the pair alone, so a thread makes those of one
// unit (W pairs) of one token and goes with them through up to eight heads.  774 MB of bf16 with pairs side by side: 287 us, 5.4 TB/s (370 us
// where a lane read two neighbouring vectors, 319 with ordinary stores); 291 MB of fp32, halves apart: 108 us, 5.4 TB/s (111 with ordinary stores).
#include "stream_common.h"

namespace dr {
namespace {

using namespace stream;

constexpr int kThreads = 256;
constexpr int64_t kCaches = 256ll << 20;  // bytes of the last-level cache

struct RopeArgs {
    const char* x;
    char* y;
    const int32_t* pos;
    int64_t pos_b, pos_axis;
    int64_t xb, xh, xn, yb, yh, yn;      // bytes
    int32_t H, N, d, units, heads;       // units of a token; heads of a thread
    float sign;
    RopeTable r;
};

// `past` the caches: a result that is larger than they are would only push other data out.
template <typename T, bool PAST>
__device__ __forceinline__ void put(char* p, const float (&x)[Pack<T>::W]) {
    typedef uint32_t v4u __attribute__((ext_vector_type(4)));
    v4u v;
    Pack<T>::store(&v, x);
    if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<v4u*>(p));
    else *reinterpret_cast<v4u*>(p) = v;
}

// One unit is two vectors of W channels: W pairs, or 2 W channels that are copied.
template <typename T, bool HALF, bool PAST>
__global__ __launch_bounds__(kThreads) void k_rope(const RopeArgs a) {
    constexpr int W = Pack<T>::W;
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int n = (int)(at / a.units), u = (int)(at - (int64_t)n * a.units);
    if (n >= a.N) return;
    const int b = blockIdx.z, h0 = blockIdx.y * a.heads, h1 = min(h0 + a.heads, a.H);
    const bool turned = 2 * W * u < a.r.dim;
    // its first vector, and the second half a row behind it, so that neighbouring lanes read neighbouring vectors; with pairs side by side the first
    // holds pairs u W / 2 .., the second dim / 4 + u W / 2 ..
    const int ca = turned ? u * W : 2 * W * u, cb = turned ? a.r.dim / 2 + u * W : ca + W;
    float c[W], s[W];
    if (turned) {
        const int32_t* p = a.pos + b * a.pos_b + n;
        int axis = -1, pos = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const int pair = HALF ? u * W + j : j < W / 2 ? u * (W / 2) + j : a.r.dim / 4 + u * (W / 2) + j - W / 2, k = rope_axis(a.r, pair);
            if (k != axis) pos = p[k * a.pos_axis];
            axis = k;
            const float2 cs = rope_cos_sin(pos, a.r.turn[pair]);
            c[j] = cs.x * (float)a.r.mscale;
            s[j] = cs.y * (float)a.r.mscale * a.sign;
        }
    }
    const char* x = a.x + b * a.xb + n * a.xn;
    char* y = a.y + b * a.yb + n * a.yn;
    for (int h = h0; h < h1; ++h) {
        const char* xr = x + h * a.xh;
        char* yr = y + h * a.yh;
        const uint4 va = *reinterpret_cast<const uint4*>(xr + ca * sizeof(T)), vb = *reinterpret_cast<const uint4*>(xr + cb * sizeof(T));
        if (!turned) {
            *reinterpret_cast<uint4*>(yr + ca * sizeof(T)) = va;
            *reinterpret_cast<uint4*>(yr + cb * sizeof(T)) = vb;
            continue;
        }
        float p[W], q[W], o[W], w[W];
        Pack<T>::load(&va, p);
        Pack<T>::load(&vb, q);
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if (HALF) {
                o[j] = p[j] * c[j] - q[j] * s[j];
                w[j] = q[j] * c[j] + p[j] * s[j];
            } else {
                const int k = j & ~1;                     // channel j of the first vector belongs to pair j / 2, of the second to (W + j) / 2
                const float e = (j & 1) ? p[k] * s[j / 2] : -p[k + 1] * s[j / 2];
                o[j] = fmaf(p[j], c[j / 2], e);
                const float f = (j & 1) ? q[k] * s[W / 2 + j / 2] : -q[k + 1] * s[W / 2 + j / 2];
                w[j] = fmaf(q[j], c[W / 2 + j / 2], f);
            }
        }
        put<T, PAST>(yr + ca * sizeof(T), o);
        put<T, PAST>(yr + cb * sizeof(T), w);
    }
}

// Any alignment and any even dim: a unit is one pair, or one channel that is copied.  37800 tokens of 20 heads of 128, 100 channels turned: bf16 190 us, 2.0 TB/s (96 of
// them in vectors: 89 us), fp32 237 us, 3.3 TB/s (144 us).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_rope_any(const RopeArgs a) {
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int n = (int)(at / a.units), u = (int)(at - (int64_t)n * a.units);
    if (n >= a.N) return;
    const int b = blockIdx.z, h0 = blockIdx.y * a.heads, h1 = min(h0 + a.heads, a.H);
    const int pairs = a.r.dim / 2;
    const char* x = a.x + b * a.xb + n * a.xn;
    char* y = a.y + b * a.yb + n * a.yn;
    if (u >= pairs) {
        const int64_t c = (int64_t)(pairs + u) * sizeof(T);
        for (int h = h0; h < h1; ++h) *reinterpret_cast<T*>(y + h * a.yh + c) = *reinterpret_cast<const T*>(x + h * a.xh + c);
        return;
    }
    const float2 cs = rope_cos_sin(a.pos[b * a.pos_b + rope_axis(a.r, u) * a.pos_axis + n], a.r.turn[u]);
    const float c = cs.x * (float)a.r.mscale, s = cs.y * (float)a.r.mscale * a.sign;
    const int64_t ca = (int64_t)(a.r.interleaved ? 2 * u : u) * sizeof(T), cb = (int64_t)(a.r.interleaved ? 2 * u + 1 : pairs + u) * sizeof(T);
    for (int h = h0; h < h1; ++h) {
        const float p = Pack<T>::one(x + h * a.xh + ca), q = Pack<T>::one(x + h * a.xh + cb);
        Pack<T>::put(y + h * a.yh + ca, p * c - q * s);
        Pack<T>::put(y + h * a.yh + cb, q * c + p * s);
    }
}

template <bool PAST>
void launch(bool bf16, const dim3& grid, const RopeArgs& a, hipStream_t st) {
    if (a.r.interleaved) {
        if (bf16) k_rope<__bf16, false, PAST><<<grid, kThreads, 0, st>>>(a);
        else k_rope<float, false, PAST><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (bf16) k_rope<__bf16, true, PAST><<<grid, kThreads, 0, st>>>(a);
        else k_rope<float, true, PAST><<<grid, kThreads, 0, st>>>(a);
    }
}

}  // namespace

hipError_t launch_rope(const RopeTensor& t, const RopeTable& r, bool bf16, const void* X, const int32_t* pos, int64_t pos_b, int64_t pos_axis,
                       void* Y, bool backward, int cus, hipStream_t st) {
    const int es = bf16 ? 2 : 4, W = 16 / es;
    RopeArgs a{};
    a.x = static_cast<const char*>(X);
    a.y = static_cast<char*>(Y);
    a.pos = pos; a.pos_b = pos_b; a.pos_axis = pos_axis;
    a.xb = t.xb * es; a.xh = t.xh * es; a.xn = t.xn * es;
    a.yb = t.yb * es; a.yh = t.yh * es; a.yn = t.yn * es;
    a.H = t.H; a.d = t.d;
    a.sign = backward ? -1.0f : 1.0f;
    a.r = r;
    const auto odd = reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(Y) | (uintptr_t)a.xb | (uintptr_t)a.xh | (uintptr_t)a.xn |
                     (uintptr_t)a.yb | (uintptr_t)a.yh | (uintptr_t)a.yn;
    const bool vec = odd % 16 == 0 && r.dim % (2 * W) == 0 && t.d % (2 * W) == 0;
    a.units = vec ? t.d / (2 * W) : r.dim / 2 + (t.d - r.dim);
    const int64_t blocks = ((int64_t)t.N * a.units + kThreads - 1) / kThreads;
    const int each = rope_tokens_of_a_launch(t.N, a.units, kThreads);
    // up to eight heads a thread share its cosines, as long as some sixteen waves a compute unit remain
    const int64_t waves = blocks * (kThreads / 64) * t.B * (int64_t)t.H;
    const int64_t most = waves / ((int64_t)cus * 16);
    a.heads = (int)(most < 1 ? 1 : most > 8 ? 8 : most);
    const bool past = (int64_t)t.B * t.H * t.N * t.d * es > kCaches;
    for (int n = 0; n < t.N; n += a.N) {
        a.N = (int)std::min<int64_t>(each, t.N - n);
        const dim3 grid((unsigned)(((int64_t)a.N * a.units + kThreads - 1) / kThreads), (unsigned)((t.H + a.heads - 1) / a.heads), (unsigned)t.B);
        if (!vec) {
            if (bf16) k_rope_any<__bf16><<<grid, kThreads, 0, st>>>(a);
            else k_rope_any<float><<<grid, kThreads, 0, st>>>(a);
        } else if (past) {
            launch<true>(bf16, grid, a, st);
        } else {
            launch<false>(bf16, grid, a, st);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.x += a.N * a.xn;
        a.y += a.N * a.yn;
        if (a.pos) a.pos += a.N;
    }
    return hipSuccess;
}

}  // namespace dr
