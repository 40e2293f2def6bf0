// The cache in 8 bits: its descriptor, where a code sits, and the conversions.  Device code shared by the append, the read-back and
// the attention of new rows.
#pragma once

#include "draft_ops.h"

namespace chiron {

constexpr int kFmtBf16 = CHIRON_BF16, kFmtInt8 = CHIRON_INT8, kFmtE4m3 = CHIRON_E4M3;

// pool over caller-owned memory: see chiron.h for the layout
struct Pool8Desc {
    uint8_t* base = nullptr;
    int64_t layer_stride = 0, exps_at = 0;  // bytes: layer to layer, and from a layer's codes to its powers of two
    int num_blocks = 0, n_kv = 0, d = 0, n_layers = 0, format = 0;
};

__device__ __forceinline__ uint8_t* tile8(const Pool8Desc& p, int layer, int block, int kvh) {
    return p.base + layer * p.layer_stride + ((int64_t)block * p.n_kv + kvh) * (32 * p.d);
}
__device__ __forceinline__ int8_t* exps8(const Pool8Desc& p, int layer, int block, int kvh) {
    return (int8_t*)p.base + layer * p.layer_stride + p.exps_at + ((int64_t)block * p.n_kv + kvh) * 2;
}
// inside a K tile, and inside a V tile
__device__ __forceinline__ int k8_off(int t, int e) { return ((e >> 4) * 16 + t) * 16 + (e & 15); }
__device__ __forceinline__ int v8_off(int t, int e) { return ((((e >> 6) * 4 + (t >> 2)) * 16 + (e & 15)) * 4 + ((e & 63) >> 4)) * 4 + (t & 3); }

constexpr int kMinExp8 = -100;            // steps are not finer than this: values stay clear of subnormal numbers (their products with weights need not)
constexpr float kLimit8 = 0x1p100f;       // and values not larger: sums of 2^27 of them are finite, with weights up to 2^8 of 2^19

__device__ __forceinline__ float bounded8(float x) {
    x = x != x ? 0.f : x;
    return fminf(fmaxf(x, -kLimit8), kLimit8);
}
// the exponent of the smallest power of two, at least 2^-100, with amax <= 127 * 2^e (448 * 2^e); 0 <= amax <= 2^100
template <int FMT>
__device__ __forceinline__ int power8(float amax) {
    if (amax == 0.f) return kMinExp8;
    const int ex = __builtin_amdgcn_frexp_expf(amax);
    const float mant = __builtin_amdgcn_frexp_mantf(amax);
    const int e = FMT == kFmtInt8 ? ex - 7 + (mant > 127.f / 128.f) : ex - 9 + (mant > 448.f / 512.f);
    return e < kMinExp8 ? kMinExp8 : e;
}
// four values, already divided by 2^e, as codes: the first in the low byte
template <int FMT>
__device__ __forceinline__ uint32_t encode8(float a, float b, float c, float d) {
    if (FMT == kFmtInt8)
        return ((uint32_t)(int)rintf(a) & 0xff) | ((uint32_t)(int)rintf(b) & 0xff) << 8 | ((uint32_t)(int)rintf(c) & 0xff) << 16 |
               (uint32_t)(int)rintf(d) << 24;
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
// the four codes of a word as fp32
template <int FMT>
__device__ __forceinline__ floatx4 decode8(uint32_t w) {
    if (FMT == kFmtInt8)
        return floatx4{(float)(int8_t)(w & 0xff), (float)(int8_t)(w >> 8 & 0xff), (float)(int8_t)(w >> 16 & 0xff), (float)((int32_t)w >> 24)};
    return floatx4{__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1), __builtin_amdgcn_cvt_f32_fp8((int)w, 2),
                   __builtin_amdgcn_cvt_f32_fp8((int)w, 3)};
}
// the four codes of a word, times a power of two, as bf16: exact in either format (int8: at most 7 significant bits and a sign)
template <int FMT>
__device__ __forceinline__ uint2 widen8(uint32_t w, float scale) {
    if (FMT == kFmtE4m3) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
        return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
    const floatx4 f = decode8<FMT>(w) * scale;
    return make_uint2(__builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302),
                      __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302));
}

}  // namespace chiron

struct chiron_kvpool8 {
    chiron::Pool8Desc d;
};
