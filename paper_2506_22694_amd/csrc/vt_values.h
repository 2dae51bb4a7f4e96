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
// x * 2^(exponent - 127) for every byte that a cache may hold: as a float's exponent bits, 0 would be no 2^-127 and 255 would make NaN of x = 0
__device__ __forceinline__ float scaled(float x, unsigned exponent) { return __builtin_ldexpf(x, (int)exponent - 127); }

}  // namespace vt
