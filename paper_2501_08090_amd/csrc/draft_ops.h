// Internal declarations of the drafting operators: page index, rotate-and-append, block-sparse attention, verification of drafts and
// 4-bit products.  They are apart from the decode step's headers, whose kernels they do not touch.
#pragma once

#include "chiron_internal.h"
#include "device_util.h"

namespace chiron {

// page index over caller-owned memory: see chiron.h for the layout
struct IndexDesc {
    int8_t* base = nullptr;
    int64_t layer_stride = 0, exps_at = 0;  // bytes: layer to layer, and from a layer's codes to its exponents
    int num_blocks = 0, n_kv = 0, d = 0, n_layers = 0;
};
IndexDesc index_layout(const PoolDesc& p);
inline bool index_fits(const IndexDesc& x, const PoolDesc& p) {
    return x.num_blocks == p.num_blocks && x.n_kv == p.n_kv && x.d == p.d && x.n_layers == p.n_layers;
}
__device__ __forceinline__ int8_t* index_codes(const IndexDesc& x, int layer, int block, int kvh) {
    return x.base + layer * x.layer_stride + ((int64_t)block * x.n_kv + kvh) * (2 * x.d);
}
__device__ __forceinline__ int8_t* index_exp(const IndexDesc& x, int layer, int block, int kvh) {
    return x.base + layer * x.layer_stride + x.exps_at + (int64_t)block * x.n_kv + kvh;
}

// exponent e of the smallest power of two, at least 2^-126, with amax <= 127 * 2^e; amax finite and >= 0
__device__ __forceinline__ int power_of(float amax) {
    if (amax == 0.f) return 0;
    const int e = __builtin_amdgcn_frexp_expf(amax) - 7 + (__builtin_amdgcn_frexp_mantf(amax) > 127.f / 128.f ? 1 : 0);
    return e < -126 ? -126 : e;
}
// 2^e, -126 <= e <= 127
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// NaN as 0, infinities as the largest value of the type
__device__ __forceinline__ float finite_or(float x, float top) {
    x = x != x ? 0.f : x;
    return fminf(fmaxf(x, -top), top);
}

// the value of the lane `Ctrl` away in the same 16 lanes (data-parallel move, one instruction)
template <int Ctrl>
__device__ __forceinline__ float row_move(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), Ctrl, 0xf, 0xf, false));
}
template <int Ctrl>
__device__ __forceinline__ int row_move(int v) {
    return __builtin_amdgcn_update_dpp(0, v, Ctrl, 0xf, 0xf, false);
}
constexpr int kRor1 = 0x121, kRor2 = 0x122, kRor4 = 0x124, kRor8 = 0x128;  // row_ror:n, rotation within 16 lanes

// a launch with dynamic LDS
template <typename... P, typename... A>
inline void launch_lds(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t st, A... args) {
    kernel<<<grid, block, lds, st>>>(static_cast<P>(args)...);
}

// device memory of a handle (api.hip)
int32_t dev_alloc(void** p, size_t bytes);

}  // namespace chiron

struct chiron_kvindex {
    chiron::IndexDesc d;
};
