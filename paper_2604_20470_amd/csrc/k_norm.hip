// Norms between the blocks of a layer, with the gated residual in front and the modulation behind, and all their gradients:
//
//   T = residual_scale X + gate b,  b = branch or norm(branch) branch_weight;  Y = norm(T) mul + add,  mul = weight (1 + scale), add = bias (1 + scale) + shift
//   norm(t) = (t - mean) r, r = 1 / sqrt(variance + eps)  (RMS: mean = 0)
//
// Back, with n = norm(T) and g = dY mul:  D = r (g - mean(g) - n mean(g n)) + dT (RMS: without mean(g));  dX = residual_scale D.  All vectors' gradients follow
// from three sums over the tokens that share a modulation, S1 = sum dY, S2 = sum dY n, S3 = sum D b' (b' = branch, or its norm):
//   dshift = S1, dscale = weight S2 + bias S1, dgate = branch_weight S3, dweight = sum (1 + scale) S2, dbias = sum (1 + scale) S1, dbranch_weight = sum gate S3,
// so a lane carries three accumulators a channel, whatever is asked for.
//
// Bound by memory: every tensor is read once and written once.  A row stays in registers, 8 channels a lane; 8 to 64 lanes of a wave have one (up to 512
// channels), or the waves of a workgroup, which then meet behind one barrier a row.  The next row is on its way while this one is reduced.  Rows of one modulation are in a row, so
// vectors are loaded when they change.  Sums over tokens leave as one partial row a piece and are added up by a second kernel, in a fixed order.
// 75600 rows of 5120 channels in bf16, branch, gate, modulation: forward 603 us, 5.1 TB/s; all gradients 982 us, 4.7 TB/s (a copy of 2 GiB: 4.8; with a barrier for every sum, and pieces
// that leave rounds of workgroups half empty, 1236).  284580 heads of 128 in fp32, gradients: 102 us, 4.3 TB/s.  48 single rows: 5.5 us, of which the loads of their vectors are most.
// 300 MB tensors of 64 to 8192 channels: 4.3 to 5.1 TB/s; bf16 rows of 5120 without a branch 4.0 and 3.6 (ten waves a workgroup leave the SIMDs uneven).  Rows that are not aligned, or whose channels do
// not come in packs: fp32 4.0 to 5.1, bf16 2.4 (few channels in the last wave) to 4.4; beyond 6144 channels back with a branch 3.1 and 3.7.
#include "norm_plan.h"
#include "stream_common.h"

#include <type_traits>

namespace dr {
namespace {

using namespace stream;

constexpr int kMaxWaves = 16;                   // of a row: 16 x 64 lanes of 8 channels

// Sum over 8 to 64 neighbouring lanes; all of them get it.
template <int G>
__device__ __forceinline__ float lanes_sum(float x) {
    auto add = [&](auto ctrl) { x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false)); };
    add(std::integral_constant<int, 0xb1>{});                                // lane ^ 1
    add(std::integral_constant<int, 0x4e>{});                                // lane ^ 2
    add(std::integral_constant<int, 0x141>{});                               // the other four of 8
    if constexpr (G > 8) add(std::integral_constant<int, 0x140>{});          // the other eight of 16
    if constexpr (G > 16) x += __shfl_xor(x, 16);
    if constexpr (G > 32) x += __shfl_xor(x, 32);
    return x;
}

// The values exist here.  Left to itself the compiler turns a row into fp32 where it needs it, behind the loads of the next one, which then go to other registers and are waited for
// to be moved (75600 rows of 5120 channels, forward: 745 us, 610 with this; in the backward pass, whose registers are scarcer, the compiler does better by itself: 977, with this 1030).
template <int E>
__device__ __forceinline__ void settle(float (&x)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) asm volatile("" : "+v"(x[e]));
}

// How the channels of a row are read: one by one (rows of fewer than a pack), in packs of 16 bytes at any address, or in packs that are aligned and whole.
enum Way { kSingle = 0, kLoose = 1, kWide = 2 };

// Packs at any address, which global memory instructions take.  Rows of 8191 channels in bf16, 300 MB a tensor, without a branch and with all there is: forward 178 and 272 us, channel by channel 200
// and 353; back 237 and 583, 328 and 1386 (more than its registers).  Of 65 channels: forward 165 and 316, 252 and 450; of 5119 the backward pass is the slower one, 319 and 574, 294 and 579.
typedef uint32_t loose4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t loose2_2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float loose4_4 __attribute__((ext_vector_type(4), aligned(4)));
template <int WAY>
__device__ __forceinline__ void get_pack(Pack<float>& v, const char* p) {
    if constexpr (WAY == kLoose) {
        const loose4_4 x = *reinterpret_cast<const loose4_4*>(p);
        v.v = make_float4(x[0], x[1], x[2], x[3]);
    } else {
        v.get(p);
    }
}
template <int WAY>
__device__ __forceinline__ void get_pack(Pack<__bf16>& v, const char* p) {
    if constexpr (WAY == kLoose) {
        const loose4_2 x = *reinterpret_cast<const loose4_2*>(p);
        v.v = make_uint4(x[0], x[1], x[2], x[3]);
    } else {
        v.get(p);
    }
}
template <int WAY>
__device__ __forceinline__ void put_pack(char* p, const float (&x)[4]) {
    if constexpr (WAY == kLoose) *reinterpret_cast<loose4_4*>(p) = loose4_4{x[0], x[1], x[2], x[3]}; else Pack<float>::store(p, x);
}
template <int WAY>
__device__ __forceinline__ void put_pack(char* p, const float (&x)[8]) {
    if constexpr (WAY == kLoose) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2bf t = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, t);
        }
        *reinterpret_cast<loose4_2*>(p) = loose4_2{w[0], w[1], w[2], w[3]};
    } else {
        Pack<__bf16>::store(p, x);
    }
}

// The E channels of a lane: packs, `lanes` packs apart.
template <typename T, int E, int WAY>
struct Slice {
    static constexpr int W = WAY != kSingle ? Pack<T>::W : 1, K = E / W;
    static constexpr bool FINE = sizeof(T) == 4;                             // means with more bits than fp32 has (see normalise)
    int lane, lanes, C;
    __device__ __forceinline__ int channel(int k) const { return (k * lanes + lane) * W; }
    __device__ __forceinline__ bool has(int e) const { return channel(e / W) + (WAY == kLoose ? e % W : 0) < C; }
    __device__ __forceinline__ int place(int k) const { return min(channel(k), C - W); }         // where pack k is read
    __device__ __forceinline__ bool whole(int k) const { return WAY != kLoose || channel(k) + W <= C; }
    // The row's last pack, if it is not whole, is read with channels in front of it: its own to the front.
    __device__ __forceinline__ void own(int k, float (&y)[W]) const {
        if constexpr (WAY == kLoose) {
            if (whole(k)) return;
            const int behind = (W - C % W) % W;
#pragma unroll
            for (int by = 1; by < W; by *= 2)
                if (behind & by) {
#pragma unroll
                    for (int j = 0; j + by < W; ++j) y[j] = y[j + by];
                }
        }
    }
    __device__ __forceinline__ int of_wave(int w) const {                    // channels that its lanes have
        int n = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) n += min(max(C - (k * lanes + 64 * w) * W, 0), 64 * W);
        return n;
    }
};
template <typename T, int E, int WAY>
struct Held {                                   // a row's channels as they were read
    using S = Slice<T, E, WAY>;
    Pack<T> v[S::K];
    __device__ __forceinline__ void load(const S& s, const char* row) {
#pragma unroll
        for (int k = 0; k < S::K; ++k) get_pack<WAY>(v[k], row + s.place(k) * (int)sizeof(T));
    }
    __device__ __forceinline__ void values(const S& s, float (&x)[E]) const {
#pragma unroll
        for (int k = 0; k < S::K; ++k) {
            float y[S::W];
            v[k].values(y);
            s.own(k, y);
#pragma unroll
            for (int j = 0; j < S::W; ++j) x[k * S::W + j] = s.has(k * S::W + j) ? y[j] : 0.0f;
        }
    }
};
template <typename T, int E>
struct Held<T, E, kSingle> {
    using S = Slice<T, E, kSingle>;
    float v[E];
    __device__ __forceinline__ void load(const S& s, const char* row) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = Pack<T>::one(row + min(s.channel(e), s.C - 1) * (int)sizeof(T));
    }
    __device__ __forceinline__ void values(const S& s, float (&x)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = s.has(e) ? v[e] : 0.0f;
    }
};
template <typename T, int E, int WAY>
__device__ __forceinline__ void put_row(const Slice<T, E, WAY>& s, char* row, const float (&x)[E]) {
    constexpr int W = Slice<T, E, WAY>::W;
#pragma unroll
    for (int k = 0; k < E / W; ++k) {
        if (s.channel(k) >= s.C) continue;
        char* at = row + s.channel(k) * (int)sizeof(T);
        if constexpr (WAY == kSingle) {
            Pack<T>::put(at, x[k]);
        } else if (s.whole(k)) {
            float y[W];
#pragma unroll
            for (int j = 0; j < W; ++j) y[j] = x[k * W + j];
            put_pack<WAY>(at, y);
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (s.has(k * W + j)) Pack<T>::put(at + j * (int)sizeof(T), x[k * W + j]);
        }
    }
}
// W channels of a vector.
template <int WAY>
__device__ __forceinline__ void vector_pack(const NormArgs& a, const char* p, int c, float (&y)[8]) {
    if (a.vector_bf16) {
        Pack<__bf16> v;
        get_pack<WAY>(v, p + c * 2);
        v.values(y);
    } else {
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            Pack<float> v;
            float z[4];
            get_pack<WAY>(v, p + (c + h) * 4);
            v.values(z);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[h + j] = z[j];
        }
    }
}
template <int WAY>
__device__ __forceinline__ void vector_pack(const NormArgs& a, const char* p, int c, float (&y)[4]) {
    if (!a.vector_bf16) {
        Pack<float> v;
        get_pack<WAY>(v, p + c * 4);
        v.values(y);
    } else if constexpr (WAY == kLoose) {
        const loose2_2 x = *reinterpret_cast<const loose2_2*>(p + c * 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = __uint_as_float(j & 1 ? x[j / 2] & 0xffff0000u : x[j / 2] << 16);
    } else {
        Four<__bf16> f;
        f.get<true>(p + c * 2);
        f.values(y);
    }
}
// A vector's channels, or `value` where there is no vector.  (One vector after another: left to itself the compiler has all of them on their way at once, in
// registers that the rows need.)
template <typename T, int E, int WAY>
__device__ __forceinline__ void get_vector(const NormArgs& a, const Slice<T, E, WAY>& s, const char* p, float value, float (&x)[E]) {
    constexpr int W = Slice<T, E, WAY>::W;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = value;
    if (!p) return;
#pragma unroll
    for (int k = 0; k < E / W; ++k) {
        if constexpr (WAY == kSingle) {
            const int c = min(s.channel(k), s.C - 1);
            x[k] = a.vector_bf16 ? Pack<__bf16>::one(p + c * 2) : Pack<float>::one(p + c * 4);
        } else {
            float y[W];
            vector_pack<WAY>(a, p, s.place(k), y);
            s.own(k, y);
#pragma unroll
            for (int j = 0; j < W; ++j) x[k * W + j] = y[j];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ const char* row_of(const NormTensor& t, int b, int n) { return t.p + (int64_t)b * t.b + (int64_t)n * t.n; }
__device__ __forceinline__ char* out_row(const NormTensor& t, int b, int n) { return t.p + (int64_t)b * t.b + (int64_t)n * t.n; }
__device__ __forceinline__ const char* mod_row(const NormTensor& t, int b, int g) { return t.p ? row_of(t, b, g) : nullptr; }

// Sums over a row: first over its part in a wave (all of it, if G lanes have it), then over the parts, through LDS, two places in turn.  One barrier is enough: nobody writes
// a place before everybody has left the barrier behind the next sum's.
template <bool FINE>
struct Place { float4 v; };
template <>
struct Place<true> { float4 v; float more; };
template <int G, bool FINE>
struct Parts {
    Place<FINE> (*lds)[kMaxWaves];
    int turn = 0;
    float mine, inverse, count;                 // channels of this wave's part, 1 / that; of part lane % 16

    template <typename S>
    __device__ __forceinline__ Parts(Place<FINE> (*places)[kMaxWaves], const S& s) : lds(places) {
        if constexpr (G != 0) return;
        const int waves = blockDim.x >> 6, part = threadIdx.x & 15;
        mine = (float)s.of_wave(threadIdx.x >> 6);
        inverse = 1.0f / fmaxf(mine, 1.0f);
        if constexpr (FINE) inverse = of_first(inverse);                     // (the same in all lanes; registers are scarce)
        count = part < waves ? (float)s.of_wave(part) : 0.0f;
        if (threadIdx.x < kMaxWaves && part >= waves) places[0][part] = places[1][part] = Place<FINE>{};
    }
    static __device__ __forceinline__ float in_wave(float x) { return lanes_sum<G ? G : 64>(x); }
    static __device__ __forceinline__ float over_parts(float x) { return G ? x : lanes_sum<16>(x); }
    // Part 0's value of what part lane % 16 has.
    static __device__ __forceinline__ float of_first(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
    // Part lane % 16's values, for all waves to sum over 16 lanes.
    template <bool MORE>
    __device__ __forceinline__ float4 meet(const float4& v, float& more) {
        if constexpr (G != 0) return v;
        if ((threadIdx.x & 63) == 0) {
            Place<FINE>& to = lds[turn][threadIdx.x >> 6];
            to.v = v;
            if constexpr (MORE) to.more = more;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // (a barrier that leaves the next row's loads and this one's stores on their way)
        const Place<FINE>& from = lds[turn][threadIdx.x & 15];
        const float4 y = from.v;
        if constexpr (MORE) more = from.more;
        turn ^= 1;
        return y;
    }
    __device__ __forceinline__ void sum2(float& x, float& y) {
        float none = 0.0f;
        const float4 v = meet<false>(make_float4(in_wave(x), in_wave(y), 0.0f, 0.0f), none);
        x = over_parts(v.x);
        y = over_parts(v.y);
    }
};

// 1 / sqrt(x), off by 2^-23 at most: the instruction's result and a step of Newton's method, where the compiler's root and division are some forty instructions.
__device__ __forceinline__ float inverse_root(float x) {
    if (!(x >= 0x1p-100f && x <= 0x1p100f)) return 1.0f / sqrtf(x);
    const float r = __builtin_amdgcn_rsqf(x);
    return fmaf(r * 0.5f, fmaf(-x * r, r, 1.0f), r);
}
// q = x / n, and the rest, for 0 <= x < 2^30: with inverse = min(2^32 / n, 2^32 - 1), the product's upper half is q or one less.
__device__ __forceinline__ int quotient(int x, int n, uint32_t inverse, int& rest) {
    int q = (int)__umulhi((uint32_t)x, inverse);
    rest = x - q * n;
    const bool more = rest >= n;
    rest -= more ? n : 0;
    return q + more;
}

// x becomes norm(x); returns 1 / deviation.  BACK: also the means of g and of g times the result.
// A part takes its own mean m first, rounded, then the sum of the distances to that, which a value near m leaves without a rounding, and of their squares (and products with g).  The sum of
// distances takes out what rounding m has left: m + o, o = sum (t - m) / n, is the part's mean with all its bits.  What comes together behind one barrier:
//   sum (t - mean)^2 = sum over parts of sum (t - m - o)^2 + n (m + o - mean)^2,  sum g (t - mean) = sum over parts of sum g (t - m - o) + (m + o - mean) sum g,
// with all means counted from the first part's m.  So in fp32 a mean far from 0 costs nothing but the roundings of t itself (rows of 5120
// at 10000 with deviation 1: off by 7e-7 at most, without o by 1.6e-3; o takes 0 to 2 % of the time, 0.5 us of a small call).
// In bf16 values that differ are 2^-8 of the mean apart, and what m loses (some 2^-23 of the mean) is some 2^-15 of a deviation, far below the result's rounding; a sum of X and branch is itself rounded to
// fp32.  So o = 0 there (with it 75 600 rows of 5120 channels take 611 us instead of 602, all their gradients 1028 instead of 994).
template <bool BACK, int G, typename S, int E>
__device__ __forceinline__ float normalise(const NormArgs& a, const S& s, Parts<G, S::FINE>& parts, float (&x)[E], const float (&g)[E], float& mean_g, float& mean_gn) {
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float each = G ? a.inv_c : parts.inverse;
    float off = 0.0f;
    if (a.layer) {
#pragma unroll
        for (int e = 0; e < E; ++e) v.x += x[e];
        v.x = parts.in_wave(v.x) * each;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        x[e] = s.has(e) ? x[e] - v.x : 0.0f;
        if constexpr (S::FINE) off += x[e];
        v.y = fmaf(x[e], x[e], v.y);
        if constexpr (BACK) {
            v.z += g[e];
            v.w = fmaf(g[e], x[e], v.w);
        }
    }
    v.y = parts.in_wave(v.y);
    if constexpr (BACK) {
        v.z = parts.in_wave(v.z);
        v.w = parts.in_wave(v.w);
    }
    if (S::FINE && a.layer) {
        const float sum = parts.in_wave(off);
        off = sum * each;
        v.y = fmaf(-off, sum, v.y);
        if constexpr (BACK) v.w = fmaf(-off, v.z, v.w);
        if constexpr (G != 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = s.has(e) ? x[e] - off : 0.0f;
        }
    }
    if constexpr (G == 0) {
        const float m = v.x;
        v = parts.template meet<S::FINE>(v, off);
        if (a.layer) {
            const float first = S::FINE ? parts.of_first(v.x) : 0.0f, at = S::FINE ? v.x - first + off : v.x;
            const float mean = parts.over_parts(parts.count * at) * a.inv_c, d = at - mean, move = S::FINE ? m - first - mean : m - mean;
            v.y = fmaf(parts.count * d, d, v.y);
            if constexpr (BACK) v.w = fmaf(d, v.z, v.w);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = s.has(e) ? x[e] + move : 0.0f;
        }
    }
    const float r = inverse_root(fmaf(parts.over_parts(v.y), a.inv_c, a.eps));
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= r;
    if constexpr (BACK) {
        mean_g = a.layer ? parts.over_parts(v.z) * a.inv_c : 0.0f;
        mean_gn = parts.over_parts(v.w) * r * a.inv_c;
    }
    return r;
}
template <int G, typename S, int E>
__device__ __forceinline__ float normalise(const NormArgs& a, const S& s, Parts<G, S::FINE>& parts, float (&x)[E]) {
    float none, none2;
    return normalise<false>(a, s, parts, x, x, none, none2);
}

template <typename T, int E, int G, int WAY, bool BRANCH, int THREADS>
__global__ __launch_bounds__(THREADS, WAY == kSingle ? 1 : sizeof(T) == 2 ? (BRANCH ? 5 : 7) : BRANCH ? 4 : 5) void k_norm_fwd(const NormArgs a) {
    constexpr bool FINE = Slice<T, E, WAY>::FINE;
    __shared__ Place<FINE> lds[2][kMaxWaves];
    const int lane = threadIdx.x & 63;
    const Slice<T, E, WAY> s{G ? lane % (G ? G : 1) : (int)threadIdx.x, G ? G : (int)blockDim.x, a.C};
    const int groups = G ? 64 / (G ? G : 1) : 1, sub = G ? lane / (G ? G : 1) : 0;
    const int64_t unit = G ? (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
    const int rows = a.B * a.N, first = (int)(unit * a.rows_each < rows ? unit * a.rows_each : rows), end = min(rows, first + a.rows_each);
    Parts<G, FINE> parts(lds, s);
    float mul[E], add[E], gate[E], bw[E];
    get_vector(a, s, a.branch_weight, 1.0f, bw);
#pragma unroll
    for (int e = 0; e < E; ++e) gate[e] = 1.0f;
    Held<T, E, WAY> x, b;
    int bn = 0, nn = 0, mod = -1;
    auto fetch = [&](int row) {                 // (behind the last row that again: no branch)
        bn = quotient(min(row, end - 1), a.N, a.inverse_n, nn);
        x.load(s, row_of(a.x, bn, nn));
        if constexpr (BRANCH) b.load(s, row_of(a.branch, bn, nn));
    };
    if (first >= end) return;
    fetch(first + sub);
    for (int base = first; base < end; base += groups) {
        const int row = base + sub, bi = bn, ni = nn;
        const bool there = row < end;
        float t[E], u[E];
        x.values(s, t);
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] *= a.residual_scale;
        settle(t);
        if constexpr (BRANCH) {
            b.values(s, u);
            settle(u);
        }
        int in_row, g = 0;
        if (a.mods) g = quotient(ni, a.mod_tokens, a.inverse_mod, in_row);
        const int now = a.mods ? bi * a.mod_rows + g : 0;
        if (there && now != mod) {
            float v[E];
            get_vector(a, s, mod_row(a.scale, bi, g), 0.0f, v);
            get_vector(a, s, a.weight, 1.0f, mul);
            get_vector(a, s, a.bias, 0.0f, add);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                mul[e] *= 1.0f + v[e];
                add[e] *= 1.0f + v[e];
            }
            get_vector(a, s, mod_row(a.shift, bi, g), 0.0f, v);
#pragma unroll
            for (int e = 0; e < E; ++e) add[e] += v[e];
            get_vector(a, s, mod_row(a.gate, bi, g), 1.0f, gate);
            mod = now;
        }
        fetch(row + groups);
        if constexpr (BRANCH) {
            if (a.branch_norm) {
                normalise(a, s, parts, u);
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] *= bw[e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = fmaf(gate[e], u[e], t[e]);
        }
        if (a.total.p && there) put_row(s, out_row(a.total, bi, ni), t);
        normalise(a, s, parts, t);
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = fmaf(t[e], mul[e], add[e]);
        if (there) put_row(s, out_row(a.y, bi, ni), t);
    }
}

// One partial row of sums, or a sum's share of a result, channel by channel.
template <typename T, int E, int WAY>
__device__ __forceinline__ void put_sums(const Slice<T, E, WAY>& s, float* row, const float (&x)[E]) {
    constexpr int W = Slice<T, E, WAY>::W;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (s.has(e)) row[s.channel(e / W) + e % W] = x[e];
}

// The same, added to what is there if there is any (each lane its own channels, run after run).
template <typename T, int E, int WAY>
__device__ __forceinline__ void add_sums(const Slice<T, E, WAY>& s, float* row, const float (&x)[E], bool more) {
    float y[E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = more && s.has(e) ? row[s.channel(e / Slice<T, E, WAY>::W) + e % Slice<T, E, WAY>::W] : 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] += x[e];
    put_sums(s, row, y);
}

// A unit (a wave, or a workgroup with G = 0) takes one piece of a run of tokens with one modulation, or several such runs whole; APART: those that share a wave have a run each, one beside the
// other (a modulation for every token, 64 channels, 30 M elements in fp32, with weight's gradient: 197 us, one run after the other 874).
template <typename T, int E, int G, int WAY, bool BRANCH, int THREADS, bool APART = false>
__global__ __launch_bounds__(THREADS, WAY == kSingle ? 1 : THREADS == 1024 || (sizeof(T) == 2 && !BRANCH) ? 4 : THREADS == 512 ? 2 : 3) void k_norm_bwd(const NormArgs a) {
    constexpr bool FINE = Slice<T, E, WAY>::FINE;
    __shared__ Place<FINE> lds[2][kMaxWaves];
    const int lane = threadIdx.x & 63;
    const Slice<T, E, WAY> s{G ? lane % (G ? G : 1) : (int)threadIdx.x, G ? G : (int)blockDim.x, a.C};
    constexpr int groups = G ? 64 / (G ? G : 1) : 1, turn = APART ? 1 : groups;
    const int side = G ? lane / (G ? G : 1) : 0, sub = APART ? 0 : side;
    const int unit = G ? (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : (int)blockIdx.x;
    Parts<G, FINE> parts(lds, s);
    const int piece = unit % a.pieces;
    const int64_t run0 = (int64_t)(unit / a.pieces) * a.runs_each, run1 = run0 + a.runs_each < a.runs ? run0 + a.runs_each : a.runs;
    float bw[E];
    get_vector(a, s, a.branch_weight, 1.0f, bw);
    for (int64_t run = run0 + (APART ? side : 0); run < run1; run += APART ? groups : 1) {
        // Tokens of the run: with modulations those of one row of them, else all tokens of all batch elements.
        const int rb = APART ? (int)((uint32_t)run / (uint32_t)a.mod_rows) : a.mods ? (int)(run / a.mod_rows) : 0;
        const int rg = APART ? (int)run - rb * a.mod_rows : a.mods ? (int)(run % a.mod_rows) : 0;
        const int n0 = a.mods ? rg * a.mod_tokens : 0, len = a.mods ? min(a.mod_tokens, a.N - n0) : a.B * a.N;
        const int first = (int)min((int64_t)len, (int64_t)piece * a.rows_each), end = (int)min((int64_t)len, (int64_t)first + a.rows_each);
        float mul[E], gate[E];
        {
            float sc[E];
            get_vector(a, s, a.weight, 1.0f, mul);
            get_vector(a, s, mod_row(a.scale, rb, rg), 0.0f, sc);
            get_vector(a, s, mod_row(a.gate, rb, rg), 1.0f, gate);
#pragma unroll
            for (int e = 0; e < E; ++e) mul[e] *= 1.0f + sc[e];
        }
        float s1[E], s2[E], s3[E];
#pragma unroll
        for (int e = 0; e < E; ++e) s1[e] = s2[e] = s3[e] = 0.0f;
        Held<T, E, WAY> t0, dy0, dt0, b0;
        int bn = 0, nn = 0;
        auto fetch = [&](int i) {               // (behind the last row that again: no branch)
            i = min(i, end - 1);
            bn = rb;
            nn = n0 + i;
            if (!a.mods) bn = quotient(i, a.N, a.inverse_n, nn);
            t0.load(s, row_of(a.x, bn, nn));
            dy0.load(s, row_of(a.y, bn, nn));
            if (a.dtotal.p) dt0.load(s, row_of(a.dtotal, bn, nn));
            if constexpr (BRANCH) b0.load(s, row_of(a.branch, bn, nn));
        };
        if (first < end) fetch(first + sub);
        for (int base = first; base < end; base += turn) {
            const int i = base + sub, bi = bn, ni = nn;
            const bool there = i < end;
            float n[E], dy[E], d[E], u[E];
            t0.values(s, n);
            dy0.values(s, dy);
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = 0.0f;
            if (a.dtotal.p) dt0.values(s, d);
            if constexpr (BRANCH) b0.values(s, u);
            fetch(i + turn);
            if (there) {
#pragma unroll
                for (int e = 0; e < E; ++e) s1[e] += dy[e];
            }
            float g[E], mean, along;
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = dy[e] * mul[e];
            const float r = normalise<true>(a, s, parts, n, g, mean, along);
            if (there) {
#pragma unroll
                for (int e = 0; e < E; ++e) s2[e] = fmaf(dy[e], n[e], s2[e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = fmaf(r, g[e] - mean - n[e] * along, d[e]);
            if (there) {
                float x[E];
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = a.residual_scale * d[e];
                put_row(s, out_row(a.dx, bi, ni), x);
            }
            if constexpr (!BRANCH) continue;
            float rbr = 1.0f;
            if (a.branch_norm) rbr = normalise(a, s, parts, u);
            if (there) {
#pragma unroll
                for (int e = 0; e < E; ++e) s3[e] = fmaf(d[e], u[e], s3[e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] *= gate[e];
            if (a.branch_norm) {
                float m = 0.0f, al = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    d[e] = s.has(e) ? d[e] * bw[e] : 0.0f;                   // (behind the last channel stands -r mean(g))
                    m += d[e];
                    al = fmaf(d[e], u[e], al);
                }
                parts.sum2(m, al);
                m = a.layer ? m * a.inv_c : 0.0f;
                al *= a.inv_c;
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = rbr * (d[e] - m - u[e] * al);
            }
            if (there && a.dbranch.p) put_row(s, out_row(a.dbranch, bi, ni), d);
        }
        if (!a.sums) continue;
        if constexpr (G != 0 && G < 64 && !APART) {       // the rows that a wave had side by side
#pragma unroll
            for (int e = 0; e < E; ++e) {
#pragma unroll
                for (int k = G; k < 64; k *= 2) {
                    s1[e] += __shfl_xor(s1[e], k);
                    s2[e] += __shfl_xor(s2[e], k);
                    s3[e] += __shfl_xor(s3[e], k);
                }
            }
        }
        if (sub != 0) continue;
        if (a.pieces > 1) {
            float* at = a.part + (run * a.pieces + piece) * 3 * a.C;
            put_sums(s, at, s1);
            put_sums(s, at + a.C, s2);
            put_sums(s, at + 2 * (int64_t)a.C, s3);
            continue;
        }
        float w[E], x[E];
        if (a.dshift.p) put_sums(s, reinterpret_cast<float*>(out_row(a.dshift, rb, rg)), s1);
        if (a.dscale.p) {
            get_vector(a, s, a.weight, 1.0f, w);
            get_vector(a, s, a.bias, 0.0f, x);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = fmaf(x[e], s1[e], w[e] * s2[e]);
            put_sums(s, reinterpret_cast<float*>(out_row(a.dscale, rb, rg)), x);
        }
        if (a.dgate.p) {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = bw[e] * s3[e];
            put_sums(s, reinterpret_cast<float*>(out_row(a.dgate, rb, rg)), x);
        }
        if (a.shares) {                         // of the vectors that all tokens have: what this unit's runs (this side's of a wave) add up to
            get_vector(a, s, mod_row(a.scale, rb, rg), 0.0f, w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                s1[e] *= 1.0f + w[e];
                s2[e] *= 1.0f + w[e];
                s3[e] *= gate[e];
            }
            const bool more = run >= run0 + (APART ? groups : 1);
            float* at = a.shares + ((int64_t)unit * (APART ? groups : 1) + (APART ? side : 0)) * 3 * a.C;
            if (a.dbias) add_sums(s, at, s1, more);
            if (a.dweight) add_sums(s, at + a.C, s2, more);
            if (a.dbranch_weight) add_sums(s, at + 2 * (int64_t)a.C, s3, more);
        }
    }
}

__device__ __forceinline__ float one_of(const NormArgs& a, const char* p, int c, float value) {
    return !p ? value : a.vector_bf16 ? Pack<__bf16>::one(p + (int64_t)c * 2) : Pack<float>::one(p + (int64_t)c * 4);
}

// Sums of `count` rows [3][C] for 32 channels: every 32nd row to a thread, eight on their way at once, then those 32 in their order.  (All three whether wanted or not would cost a
// norm of heads, with one, 40 us instead of 10.)
__device__ __forceinline__ bool rows_sum(const NormArgs& a, const float* rows, int64_t count, const bool (&wanted)[3], float (&v)[3]) {
    __shared__ float lds[3][32][33];
    constexpr int AHEAD = 8;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        float t = 0.0f;
        if (wanted[j] && c < a.C)
            for (int64_t i = y; i < count; i += 32 * AHEAD) {
                float z[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) z[k] = i + 32 * k < count ? rows[((i + 32 * k) * 3 + j) * a.C + c] : 0.0f;
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) t += z[k];
            }
        lds[j][y][x] = t;
    }
    __syncthreads();
    if (y != 0 || c >= a.C) return false;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        v[j] = 0.0f;
        for (int i = 0; i < 32; ++i) v[j] += lds[j][i][x];
    }
    return true;
}
__device__ __forceinline__ void put_shares(const NormArgs& a, int c, const float (&v)[3]) {
    if (a.dbias) a.dbias[c] = v[0];
    if (a.dweight) a.dweight[c] = v[1];
    if (a.dbranch_weight) a.dbranch_weight[c] = v[2];
}

// The pieces of run blockIdx.y: the gradients of its modulation, and its share of the vectors that all tokens have.
__global__ __launch_bounds__(1024) void k_norm_runs(const NormArgs a) {
    const int run = blockIdx.y, c = blockIdx.x * 32 + (threadIdx.x & 31);
    const bool wanted[3] = {a.dshift.p || a.dbias || (a.dscale.p && a.bias), a.dscale.p || a.dweight, a.dgate.p || a.dbranch_weight};
    float v[3];
    if (!rows_sum(a, a.part + (int64_t)run * a.pieces * 3 * a.C, a.pieces, wanted, v)) return;
    const int b = a.mods ? run / a.mod_rows : 0, g = a.mods ? run % a.mod_rows : 0;
    if (a.dshift.p) reinterpret_cast<float*>(out_row(a.dshift, b, g))[c] = v[0];
    if (a.dscale.p) reinterpret_cast<float*>(out_row(a.dscale, b, g))[c] = fmaf(one_of(a, a.bias, c, 0.0f), v[0], one_of(a, a.weight, c, 1.0f) * v[1]);
    if (a.dgate.p) reinterpret_cast<float*>(out_row(a.dgate, b, g))[c] = one_of(a, a.branch_weight, c, 1.0f) * v[2];
    if (!a.dbias && !a.dweight && !a.dbranch_weight) return;
    const float sc = 1.0f + one_of(a, mod_row(a.scale, b, g), c, 0.0f);
    v[0] *= sc;
    v[1] *= sc;
    v[2] *= one_of(a, mod_row(a.gate, b, g), c, 1.0f);
    if (a.runs == 1) return put_shares(a, c, v);
#pragma unroll
    for (int j = 0; j < 3; ++j) a.shares[((int64_t)run * 3 + j) * a.C + c] = v[j];
}
// Shares from, from + each, ... of blockIdx.y added up, into `to`, or (to = NULL) the results.
__global__ __launch_bounds__(1024) void k_norm_shares(const NormArgs a, const float* from, int64_t count, int64_t each, float* to) {
    const int64_t at = blockIdx.y * each;
    const int c = blockIdx.x * 32 + (threadIdx.x & 31);
    const bool wanted[3] = {a.dbias != nullptr, a.dweight != nullptr, a.dbranch_weight != nullptr};
    float v[3];
    if (!rows_sum(a, from + at * 3 * a.C, count - at < each ? count - at : each, wanted, v)) return;
    if (!to) return put_shares(a, c, v);
#pragma unroll
    for (int j = 0; j < 3; ++j) to[((int64_t)blockIdx.y * 3 + j) * a.C + c] = v[j];
}

__global__ __launch_bounds__(256) void k_norm_zero(const NormArgs a) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    const float v[3] = {0.0f, 0.0f, 0.0f};
    if (c < a.C) put_shares(a, c, v);
}

struct Shape { int G, threads; };
Shape shape_of(int C) {
    if (C <= 512) return {C <= 64 ? 8 : C <= 128 ? 16 : C <= 256 ? 32 : 64, 256};
    return {0, (C + 511) / 512 * 64};
}
// Units (waves, or workgroups with G = 0) that the device holds at once, by the waves of a SIMD that registers allow.
int64_t units_at_once(const Shape& s, int waves, int cus) { return (int64_t)cus * (s.G ? 4 * waves : std::max(1, 256 * waves / s.threads)); }

template <bool BWD, typename T, int G, int WAY, int THREADS>
void launch(const NormArgs& a, unsigned grid, int threads, hipStream_t st) {
    if constexpr (BWD) {
        // (With a branch, 8192 channels in fp32: 16 channels a lane, in half as many lanes with twice the registers, 836 us where 8 and 1024 threads take 922.)
        if constexpr (G != 0 && G < 64) {
            if (a.apart) {
                if (a.branch.p) k_norm_bwd<T, 8, G, WAY, true, THREADS, true><<<grid, threads, 0, st>>>(a);
                else k_norm_bwd<T, 8, G, WAY, false, THREADS, true><<<grid, threads, 0, st>>>(a);
                return;
            }
        }
        constexpr bool FEW = WAY != kSingle && THREADS == 1024 && sizeof(T) == 4;
        if (!a.branch.p) k_norm_bwd<T, 8, G, WAY, false, THREADS><<<grid, threads, 0, st>>>(a);
        else if constexpr (FEW) k_norm_bwd<T, 16, G, WAY, true, 512><<<grid, (a.C + 1023) / 1024 * 64, 0, st>>>(a);
        else k_norm_bwd<T, 8, G, WAY, true, THREADS><<<grid, threads, 0, st>>>(a);
    } else {
        if (a.branch.p) k_norm_fwd<T, 8, G, WAY, true, THREADS><<<grid, threads, 0, st>>>(a);
        else k_norm_fwd<T, 8, G, WAY, false, THREADS><<<grid, threads, 0, st>>>(a);
    }
}
template <bool BWD, typename T, int WAY>
void launch_shape(const NormArgs& a, const Shape& s, unsigned grid, hipStream_t st) {
    if (WAY == kSingle || s.G == 8) return launch<BWD, T, 8, WAY, 256>(a, grid, s.threads, st);
    if constexpr (WAY != kSingle) {
        if (s.G == 16) launch<BWD, T, 16, WAY, 256>(a, grid, s.threads, st);
        else if (s.G == 32) launch<BWD, T, 32, WAY, 256>(a, grid, s.threads, st);
        else if (s.G == 64) launch<BWD, T, 64, WAY, 256>(a, grid, s.threads, st);
        else if (s.threads <= 768) launch<BWD, T, 0, WAY, 768>(a, grid, s.threads, st);      // (the registers of three waves a SIMD)
        else launch<BWD, T, 0, WAY, 1024>(a, grid, s.threads, st);
    }
}
template <bool BWD, typename T>
void launch_way(const NormArgs& a, const Shape& s, unsigned grid, hipStream_t st) {
    if (a.wide) launch_shape<BWD, T, kWide>(a, s, grid, st);
    else if (a.C >= Pack<T>::W) launch_shape<BWD, T, kLoose>(a, s, grid, st);
    else launch_shape<BWD, T, kSingle>(a, s, grid, st);
}
template <bool BWD>
void launch_type(const NormArgs& a, const Shape& s, unsigned grid, hipStream_t st) {
    a.bf16 ? launch_way<BWD, __bf16>(a, s, grid, st) : launch_way<BWD, float>(a, s, grid, st);
}

// Rows of one workgroup of k_norm_shares (a launch has fewer than 2^16 along an axis).
int64_t share_rows(int64_t rows) { return std::max<int64_t>(1024, (rows + 32767) / 32768); }

}  // namespace

hipError_t launch_norm_fwd(NormArgs a, int cus, hipStream_t st) {
    const Shape s = shape_of(a.C);
    const int64_t rows = (int64_t)a.B * a.N, slots = units_at_once(s, a.bf16 ? (a.branch.p ? 5 : 7) : a.branch.p ? 4 : 5, cus);
    const int groups = s.G ? 64 / s.G : 1;
    // Whole rounds of units, of some 20 turns each.
    const int64_t turns = (rows + groups - 1) / groups, rounds = std::max<int64_t>(1, turns / (20 * slots));
    a.rows_each = (int)((turns + rounds * slots - 1) / (rounds * slots)) * groups;
    const int64_t used = (rows + a.rows_each - 1) / a.rows_each;
    launch_type<false>(a, s, (unsigned)(s.G ? (used + 3) / 4 : used), st);
    return hipGetLastError();
}

NormPlan norm_plan(const NormArgs& a, int cus) {
    const Shape s = shape_of(a.C);
    NormPlan p{};
    p.runs = a.mods ? (int64_t)a.B * a.mod_rows : 1;
    const int64_t length = a.mods ? std::min(a.mod_tokens, a.N) : (int64_t)a.B * a.N;
    const int groups = s.G ? 64 / s.G : 1;
    const int64_t slots = units_at_once(s, a.bf16 && !a.branch.p ? 4 : 3, cus), turns = (length + groups - 1) / groups;
    const NormPieces cut = norm_pieces(p.runs, turns, slots);
    p.pieces = (int)cut.pieces;
    p.rows_each = (int)((turns + p.pieces - 1) / p.pieces) * groups;
    p.pieces = (int)((length + p.rows_each - 1) / p.rows_each);
    p.runs_each = p.pieces > 1 ? 1 : (int)((p.runs + 4 * slots - 1) / (4 * slots));
    // Runs side by side in a wave, where its turns would be mostly empty (30 M elements in fp32, 3 tokens to a modulation, weight's gradient too: 64 channels 123 us, one run after the other 321; 256 channels 123 and 148).
    const int64_t sides = (p.runs + groups - 1) / groups;
    if (a.mods && p.pieces == 1 && length < 2 * groups && groups > 1 && (double)((sides + slots - 1) / slots) * (double)(length + 8) < cut.time) {
        p.apart = true;
        p.runs_each = (int)((sides + 4 * slots - 1) / (4 * slots)) * groups;
    }
    const bool shares = a.dweight || a.dbias || a.dbranch_weight, sums = shares || a.dgate.p || a.dscale.p || a.dshift.p;
    const size_t row = 3 * sizeof(float) * a.C;
    if (sums && p.pieces > 1) p.part = (size_t)p.runs * p.pieces * row;
    if (shares && (p.runs > 1 || p.pieces == 1)) {
        // A row of shares for each run that is cut into pieces, else for each unit (each side of a wave): the scratch is bounded by the device, not by the tokens.
        const int64_t units = (p.runs + p.runs_each - 1) / p.runs_each, last = p.runs - (units - 1) * p.runs_each;
        p.rows = p.pieces > 1 ? p.runs : p.apart ? (units - 1) * groups + std::min<int64_t>(groups, last) : units;
        p.shares = (size_t)(p.rows + (p.rows + share_rows(p.rows) - 1) / share_rows(p.rows)) * row;
    }
    p.sums = sums;
    return p;
}

hipError_t launch_norm_bwd(NormArgs a, const NormPlan& p, void* scratch, hipStream_t st) {
    const Shape s = shape_of(a.C);
    a.runs = p.runs;
    a.pieces = p.pieces;
    a.rows_each = p.rows_each;
    a.runs_each = p.runs_each;
    a.apart = p.apart;
    a.sums = p.sums;
    a.part = static_cast<float*>(scratch);
    a.shares = p.shares ? reinterpret_cast<float*>(static_cast<char*>(scratch) + p.part) : nullptr;
    const int64_t units = p.pieces > 1 ? p.runs * p.pieces : (p.runs + p.runs_each - 1) / p.runs_each;
    launch_type<true>(a, s, (unsigned)(s.G ? (units + 3) / 4 : units), st);
    const unsigned tiles = (unsigned)((a.C + 31) / 32);
    if (p.part) k_norm_runs<<<dim3(tiles, (unsigned)p.runs), 1024, 0, st>>>(a);
    if (p.shares) {
        const int64_t each = share_rows(p.rows), chunks = (p.rows + each - 1) / each;
        float* more = a.shares + p.rows * 3 * a.C;
        k_norm_shares<<<dim3(tiles, (unsigned)chunks), 1024, 0, st>>>(a, a.shares, p.rows, each, chunks > 1 ? more : nullptr);
        if (chunks > 1) k_norm_shares<<<dim3(tiles, 1), 1024, 0, st>>>(a, more, chunks, chunks, nullptr);
    }
    return hipGetLastError();
}

hipError_t launch_norm_zero(const NormArgs& a, hipStream_t st) {
    k_norm_zero<<<(a.C + 255) / 256, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace dr
