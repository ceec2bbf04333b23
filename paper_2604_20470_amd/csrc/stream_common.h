// Device helpers shared by the streaming operators (rotary positions, paged cache): angles in fixed point, the places of a
// ragged batch, e4m3 rounding.  Internal: not part of the public ABI.
#pragma once

#include "dr_internal.h"

namespace dr {
namespace stream {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// cos and sin of position * f.  `turn` holds 2^64 * f / 2 pi, so the product modulo 2^64 is the angle's fraction of a turn however far
// the position is: nothing is lost to a range reduction.  Its upper 32 bits are kept (2^-32 of a turn); less than an eighth of a turn
// from the nearest quarter remains for two Taylor polynomials in fp32 (truncated at 2e-9 and 5e-10).
__device__ __forceinline__ float2 rope_cos_sin(int32_t pos, uint64_t turn) {
    const uint32_t lo = (uint32_t)turn, hi = (uint32_t)(turn >> 32), p = (uint32_t)pos;
    uint32_t t = __umulhi(p, lo) + p * hi;
    if (pos < 0) t -= lo;
    t += 0x20000000u;                                                        // an eighth of a turn
    const uint32_t quarter = t >> 30;
    const float x = (float)((int32_t)(t & 0x3fffffffu) - 0x20000000) * (float)(6.283185307179586476925 / 4294967296.0);
    const float xx = x * x;
    float s = fmaf(xx, 1.0f / 362880.0f, -1.0f / 5040.0f);
    s = fmaf(s, xx, 1.0f / 120.0f);
    s = fmaf(s, xx, -1.0f / 6.0f);
    s = fmaf(s * xx, x, x);
    float c = fmaf(xx, -1.0f / 3628800.0f, 1.0f / 40320.0f);
    c = fmaf(c, xx, -1.0f / 720.0f);
    c = fmaf(c, xx, 1.0f / 24.0f);
    c = fmaf(c, xx, -0.5f);
    c = fmaf(c, xx, 1.0f);
    const float a = (quarter & 1) ? s : c, b = (quarter & 1) ? c : s;        // |cos|, |sin|
    return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}
__device__ __forceinline__ int rope_axis(const RopeTable& r, int pair) { return pair_axis(r.end0, r.end1, pair); }

template <typename T> struct Pack;                                           // 16 bytes of T
template <> struct Pack<float> {
    static constexpr int W = 4;
    float4 v;
    __device__ __forceinline__ void get(const void* p) { v = *static_cast<const float4*>(p); }
    __device__ __forceinline__ void values(float (&x)[4]) const { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    static __device__ __forceinline__ void load(const void* p, float (&x)[4]) {
        Pack a;
        a.get(p);
        a.values(x);
    }
    static __device__ __forceinline__ void store(void* p, const float (&x)[4]) { *static_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
    static __device__ __forceinline__ float one(const void* p) { return *static_cast<const float*>(p); }
    static __device__ __forceinline__ void put(void* p, float x) { *static_cast<float*>(p) = x; }
};
template <> struct Pack<__bf16> {
    static constexpr int W = 8;
    uint4 v;
    __device__ __forceinline__ void get(const void* p) { v = *static_cast<const uint4*>(p); }
    __device__ __forceinline__ void values(float (&x)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void load(const void* p, float (&x)[8]) {
        Pack a;
        a.get(p);
        a.values(x);
    }
    static __device__ __forceinline__ void store(void* p, const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2bf t = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, t);
        }
        *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float one(const void* p) { return __uint_as_float((uint32_t) * static_cast<const uint16_t*>(p) << 16); }
    static __device__ __forceinline__ void put(void* p, float x) { *static_cast<__bf16*>(p) = (__bf16)x; }
};

template <typename T> struct Four;                                           // four values in a row, in a vector or (odd addresses) one by one
template <> struct Four<float> {
    float4 v;
    template <bool VEC>
    __device__ __forceinline__ void get(const void* p) {
        const float* x = static_cast<const float*>(p);
        v = VEC ? *static_cast<const float4*>(p) : make_float4(x[0], x[1], x[2], x[3]);
    }
    __device__ __forceinline__ void keep(bool k) { v = k ? v : make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void values(float (&x)[4]) const { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
};
template <> struct Four<__bf16> {
    uint2 v;
    template <bool VEC>
    __device__ __forceinline__ void get(const void* p) {
        const uint16_t* x = static_cast<const uint16_t*>(p);
        v = VEC ? *static_cast<const uint2*>(p) : make_uint2(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16);
    }
    __device__ __forceinline__ void keep(bool k) { v = k ? v : make_uint2(0u, 0u); }
    __device__ __forceinline__ void values(float (&x)[4]) const {
        x[0] = __uint_as_float(v.x << 16);
        x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16);
        x[3] = __uint_as_float(v.y & 0xffff0000u);
    }
};

// The sequence of a work item, by a search of 64 at a time; called by whole waves.
__device__ __forceinline__ Place find_place(const BatchArgs& b, int item, int mul, int tile, int slack) {
    const int lane = threadIdx.x & 63;
    return place_of(b, item, mul, tile, slack, [&](int lo, int step, int hi) {
        const int64_t i = lo + (int64_t)lane * step;
        return (int)__popcll(__ballot(i < hi && batch_first(b, i < hi ? (int)i : 0, mul, tile, slack) <= item));
    });
}

__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }     // -126 <= e <= 127

// Four values to e4m3 codes, nearest even: at most 448, or NaN (which stays).
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ float saturate(float x) { return fabsf(x) > 448.0f ? copysignf(448.0f, x) : x; }   // (false for NaN)

}  // namespace stream
}  // namespace dr
