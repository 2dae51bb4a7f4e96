// Vectors of bf16 / fp32 / e4m3 values as floats, and sums over the lanes that share a head.
#pragma once
#include "vt_attn.h"
#include "vt_cells.h"
#include "vt_device.h"

namespace vt {

typedef __attribute__((ext_vector_type(4))) float f32x4v;

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
    bf16x2 r = {(__bf16)a, (__bf16)b};      // round to nearest even
    return __builtin_bit_cast(unsigned, r);
}
__device__ __forceinline__ float low_bf16(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high_bf16(unsigned u) { return __uint_as_float(u & 0xFFFF0000u); }

struct Bf16 {
    typedef uint16_t store;
    typedef u32x2 raw4;      // four values as they are stored
    static __device__ __forceinline__ void open4(raw4 u, float *x) {
        x[0] = low_bf16(u.x), x[1] = high_bf16(u.x), x[2] = low_bf16(u.y), x[3] = high_bf16(u.y);
    }
    static __device__ __forceinline__ void load4(const store *p, float *x) { open4(*reinterpret_cast<const raw4 *>(p), x); }
    static __device__ __forceinline__ void store4(store *p, const float *x) {
        *reinterpret_cast<u32x2 *>(p) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    }
    // ... past the caches' order of use: what a kernel writes once and does not read
    static __device__ __forceinline__ void stream4(store *p, const float *x) {
        __builtin_nontemporal_store(u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])}, reinterpret_cast<u32x2 *>(p));
    }
};
struct F32 {
    typedef float store;
    typedef f32x4v raw4;
    static __device__ __forceinline__ void open4(raw4 u, float *x) { x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w; }
    static __device__ __forceinline__ void load4(const store *p, float *x) { open4(*reinterpret_cast<const raw4 *>(p), x); }
    static __device__ __forceinline__ void store4(store *p, const float *x) {
        *reinterpret_cast<f32x4v *>(p) = f32x4v{x[0], x[1], x[2], x[3]};
    }
    static __device__ __forceinline__ void stream4(store *p, const float *x) {
        __builtin_nontemporal_store(f32x4v{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4v *>(p));
    }
};

// Sum / maximum over groups of GL = 8, 16 or 32 neighbouring lanes; every lane of a group receives it.
template <int GL, typename Op>
__device__ __forceinline__ float group_reduce(float v, Op op) {
    unsigned u = __float_as_uint(v);
    u = op(u, dpp_mov<0xB1>(u));
    u = op(u, dpp_mov<0x4E>(u));
    u = op(u, dpp_mov<0x141>(u));
    if constexpr (GL >= 16) u = op(u, dpp_mov<0x140>(u));
    if constexpr (GL >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        u = op(r[0], r[1]);
    }
    return __uint_as_float(u);
}
template <int GL>
__device__ __forceinline__ float group_sum(float v) {
    return group_reduce<GL>(v, OpAddF32{});
}
// ... of 64 bits
template <int GL>
__device__ __forceinline__ double group_sum(double v) {
    auto part = [](double x, int high) { return (unsigned)(__double_as_longlong(x) >> (32 * high)); };
    auto whole = [](unsigned lo, unsigned hi) { return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo)); };
    v += whole(dpp_mov<0xB1>(part(v, 0)), dpp_mov<0xB1>(part(v, 1)));
    v += whole(dpp_mov<0x4E>(part(v, 0)), dpp_mov<0x4E>(part(v, 1)));
    v += whole(dpp_mov<0x141>(part(v, 0)), dpp_mov<0x141>(part(v, 1)));
    if constexpr (GL >= 16) v += whole(dpp_mov<0x140>(part(v, 0)), dpp_mov<0x140>(part(v, 1)));
    if constexpr (GL >= 32) {
        const auto lo = __builtin_amdgcn_permlane16_swap(part(v, 0), part(v, 0), false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(part(v, 1), part(v, 1), false, false);
        v = whole(lo[0], hi[0]) + whole(lo[1], hi[1]);
    }
    return v;
}
template <int GL>
__device__ __forceinline__ float group_max(float v) {
    return group_reduce<GL>(v, OpMaxF32{});
}

__device__ __forceinline__ int64_t index_at(const IndexArgs &a, int64_t i) {
    return a.wide ? static_cast<const int64_t *>(a.p)[i] : (int64_t) static_cast<const int32_t *>(a.p)[i];
}

// Four values as e4m3 codes of the scale whose inverse is given.  The clamp keeps what is infinite at the largest code, `most`; NaN stays
// NaN.
__device__ __forceinline__ unsigned pack_e4m3(const float *x, float inverse, float most) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i] = x[i] * inverse;
        const float c = __builtin_amdgcn_fmed3f(y[i], -most, most);
        y[i] = y[i] != y[i] ? y[i] : c;
    }
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], u, true);
}
// A value of 64 bits as one of fp32 that any further rounding takes for the value itself: cut off, and odd where something was cut off, so that it lies
// on the same side of every border and is on one only if the value is.
__device__ __forceinline__ float round_to_odd(double x) {
    const float f = (float)x;
    unsigned u = __float_as_uint(f);
    u -= fabs((double)f) > fabs(x) ? 1u : 0u;
    return __uint_as_float((double)__uint_as_float(u) != x ? u | 1u : u);
}
// Eight values as 4-bit codes of the scale 2^(exponent - 127), the first one lowest.  (The conversion takes infinities and what is past 6 for 6.  With the
// scale of the largest fp32 values 4 would be infinite: at most 3 there.)
__device__ __forceinline__ unsigned pack_e2m1(const float *x, int exponent) {
    const float most = exponent == 253 ? 3.0f * 0x1p126f : __FLT_MAX__, scale = __uint_as_float((unsigned)exponent << 23);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -most, most);
    unsigned u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], scale, 0);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[2], y[3], scale, 1);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[4], y[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[6], y[7], scale, 3);
}
// The codes as values.  Scale 255 stands for NaN, which the conversion makes of it.
__device__ __forceinline__ void open_e2m1(unsigned u, unsigned exponent, float *x) {
    const float scale = __uint_as_float(exponent << 23);
    typedef __attribute__((ext_vector_type(2))) float f32x2v;
    const f32x2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 1);
    const f32x2v c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 3);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
}
// x * 2^(exponent - 127) for every byte that a cache may hold: as a float's exponent bits, 0 would be no 2^-127 and 255 would make NaN of x = 0
__device__ __forceinline__ float scaled(float x, unsigned exponent) { return __builtin_ldexpf(x, (int)exponent - 127); }

}  // namespace vt
