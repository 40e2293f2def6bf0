// Products of few rows with 4-bit weights: y = x W^T, W[n][k] = (w4 - z) * scale, a scale and a zero point for each row and group of
// 32, 64 or 128 inputs.  gfx950, wave64.
//
// Within a group the product is whole-number arithmetic on the 8-bit matrix cores.  A weight enters as 16 * (w4 - 8), which is its
// four bits (with the highest one inverted, done when the matrix is laid out) moved to the upper half of a byte: two instructions for
// four weights.  x enters, per row and group, as whole multiples of a power of two, |x| <= 2^22, in three signed 8-bit digits.  A
// group's digit sums are exact; they are scaled and added over the groups in fp32.
//
// Layout: tiles of 16 rows of W and 128 of K, 1 KiB each: lane l holds row l % 16 and 32 values of K in one 16-byte load, two dwords
// for each step of 64.  Within a step byte j of lane group g is k = 32 * (j / 8) + 8 g + j % 8, for W and x alike, so that a group of
// 32 is what the halves of the operand registers hold.
#include <new>

#include "draft_ops.h"

namespace chiron {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct Linear4 {
    uint8_t* w = nullptr;      // [N/16][K/128][64 lanes][16 B]
    uint16_t* scale = nullptr; // [N/16][groups][16] bf16
    int8_t* zero = nullptr;    // [N/16][groups][16] z - 8, or null
    int N = 0, K = 0, group = 0, Kpad = 0, groups = 0;  // groups: of Kpad
};

// ---- laying out ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pack4_kernel(const uint8_t* __restrict__ w4, Linear4 l) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;  // (tile, block of 128, lane)
    const int kb = l.Kpad / 128;
    const int lane = (int)(j & 63);
    const int64_t tb = j >> 6;
    const int64_t tile = tb / kb;
    const int b = (int)(tb % kb);
    if (tile * 16 >= l.N) return;
    const int64_t n = tile * 16 + (lane & 15);
    const int g = lane >> 4;
    uint32_t out[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) {  // dword d: 8 values from this k on
        const int k0 = b * 128 + d / 2 * 64 + d % 2 * 32 + g * 8;
        uint32_t v = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = k0 + i;
            uint32_t q = 8;  // outside: weight 0
            if (n < l.N && k < l.K) {
                const uint8_t two = w4[n * (l.K / 2) + k / 2];
                q = (k & 1) ? two >> 4 : two & 15;
            }
            v |= (q ^ 8) << (i < 4 ? 8 * i + 4 : 8 * (i - 4));  // the first four in the upper halves of the bytes
        }
        out[d] = v;
    }
    *reinterpret_cast<uint4*>(l.w + j * 16) = make_uint4(out[0], out[1], out[2], out[3]);
}

__global__ __launch_bounds__(256) void pack4_scales_kernel(const uint16_t* __restrict__ scales, const uint8_t* __restrict__ zeros, Linear4 l) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;  // (tile, group, row)
    const int64_t tile = j / (16 * (int64_t)l.groups);
    const int64_t n = tile * 16 + (j & 15);
    const int g = (int)(j / 16 % l.groups), live = l.K / l.group;
    if (tile * 16 >= l.N) return;
    const bool there = n < l.N && g < live;
    l.scale[j] = there ? scales[n * live + g] : 0;
    if (l.zero) l.zero[j] = there ? (int8_t)((int)(zeros[n * live + g] & 15) - 8) : 0;
}

// ---- x as digits -----------------------------------------------------------------------------------------------
// digits [rows/16][Kpad/64][3][64 lanes][16 B], scales [rows/16][groups][16] fp32, digit sums [rows/16][groups][3][16] int32 (for zero points)
struct Digits {
    uint8_t* d = nullptr;
    float* scale = nullptr;
    int32_t* sum = nullptr;
};
// one wave per (16 rows, 128 of K)
__global__ __launch_bounds__(64) void digits_kernel(const float* __restrict__ x, int M, Linear4 l, Digits dg) {
    const int b = blockIdx.x, mt = blockIdx.y, lane = threadIdx.x, g = lane >> 4, kb = l.Kpad / 128;
    const int64_t m = (int64_t)mt * 16 + (lane & 15);
    float v[4][8];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int k0 = b * 128 + d / 2 * 64 + d % 2 * 32 + g * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[d][i] = m < M && k0 + i < l.K ? x[m * l.K + k0 + i] : 0.f;
    }
    // the largest magnitude of each 32: as bits, so that infinities and NaN come out on top
    uint32_t top[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        top[d] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top[d] = max(top[d], __float_as_uint(v[d][i]) & 0x7fffffffu);
        top[d] = max(top[d], (uint32_t)__shfl_xor((int)top[d], 16));
        top[d] = max(top[d], (uint32_t)__shfl_xor((int)top[d], 32));
    }
    if (l.group >= 64) {
        top[0] = top[1] = max(top[0], top[1]);
        top[2] = top[3] = max(top[2], top[3]);
    }
    if (l.group == 128) top[0] = top[1] = top[2] = top[3] = max(top[0], top[2]);
    uint32_t out[3][4][2];
    int sum[4][3];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const bool bad = top[d] >= 0x7f800000u;
        const int ex = bad ? 0 : __builtin_amdgcn_frexp_expf(__uint_as_float(top[d]));
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            out[t][d][0] = out[t][d][1] = 0;
            sum[d][t] = 0;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int q = bad ? 0 : (int)rintf(ldexpf(v[d][i], 22 - ex));
            const int d0 = (int8_t)q;
            q = (q - d0) >> 8;
            const int d1 = (int8_t)q;
            const int d2 = (q - d1) >> 8;
            out[0][d][i / 4] |= (uint32_t)(d0 & 255) << (8 * (i & 3));
            out[1][d][i / 4] |= (uint32_t)(d1 & 255) << (8 * (i & 3));
            out[2][d][i / 4] |= (uint32_t)(d2 & 255) << (8 * (i & 3));
            sum[d][0] += d0;
            sum[d][1] += d1;
            sum[d][2] += d2;
        }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < 3; ++t)
            *reinterpret_cast<uint4*>(dg.d + ((((int64_t)mt * (kb * 2) + b * 2 + s) * 3 + t) * 64 + lane) * 16) =
                make_uint4(out[t][2 * s][0], out[t][2 * s][1], out[t][2 * s + 1][0], out[t][2 * s + 1][1]);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            sum[d][t] += __shfl_xor(sum[d][t], 16);
            sum[d][t] += __shfl_xor(sum[d][t], 32);
        }
    if (lane < 16) {
        const int per = 128 / l.group;
        for (int u = 0; u < per; ++u) {
            const int d0 = u * (4 / per);
            const int64_t at = (int64_t)mt * l.groups + b * per + u;
            const bool bad = top[d0] >= 0x7f800000u;
            const int ex = bad ? 0 : __builtin_amdgcn_frexp_expf(__uint_as_float(top[d0]));
            dg.scale[at * 16 + lane] = bad ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, ex - 26);  // 2^-22, and 2^-4 of the weights
            if (dg.sum)
                for (int t = 0; t < 3; ++t) {
                    int v2 = 0;
                    for (int d = 0; d < 4 / per; ++d) v2 += sum[d0 + d][t];
                    dg.sum[(at * 3 + t) * 16 + lane] = v2;
                }
        }
    }
}

// ---- the product -----------------------------------------------------------------------------------------------
// A wave owns 16 columns (rows of W) and 16 rows of x over the whole of K.
template <int GROUP, bool ZERO>
__global__ __launch_bounds__(256) void linear4_kernel(Linear4 l, Digits dg, int M, float* __restrict__ y, int accumulate) {
    const int lane = threadIdx.x & 63, g4 = lane >> 4;
    const int tile = blockIdx.x * 4 + (threadIdx.x >> 6), mt = blockIdx.y, kb = l.Kpad / 128;
    if (tile * 16 >= l.N) return;
    const uint8_t* wp = l.w + ((int64_t)tile * kb * 64 + lane) * 16;
    const uint8_t* xp = dg.d + ((int64_t)mt * kb * 6 * 64 + lane) * 16;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int PER = 128 / GROUP;
    for (int b = 0; b < kb; ++b) {
        const uint4 w = *reinterpret_cast<const uint4*>(wp + (int64_t)b * 1024);
        const uint32_t wd[4] = {w.x, w.y, w.z, w.w};
        intx4 a[2];  // bytes: the upper halves of the dword's bytes, then the lower ones
#pragma unroll
        for (int s = 0; s < 2; ++s)
            a[s] = intx4{(int)(wd[2 * s] & 0xf0f0f0f0u), (int)((wd[2 * s] << 4) & 0xf0f0f0f0u), (int)(wd[2 * s + 1] & 0xf0f0f0f0u),
                         (int)((wd[2 * s + 1] << 4) & 0xf0f0f0f0u)};
        intx4 xd[2][3];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 3; ++t) xd[s][t] = *reinterpret_cast<const intx4*>(xp + ((int64_t)(b * 2 + s) * 3 + t) * 1024);
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            intx4 p[3];
#pragma unroll
            for (int t = 0; t < 3; ++t) {
                p[t] = intx4{0, 0, 0, 0};
                if constexpr (GROUP == 128) {
                    p[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[0], xd[0][t], p[t], 0, 0, 0);
                    p[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[1], xd[1][t], p[t], 0, 0, 0);
                } else if constexpr (GROUP == 64) {
                    p[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u], xd[u][t], p[t], 0, 0, 0);
                } else {
                    const int h = (u & 1) * 2;
                    const int64_t av = (uint32_t)a[u / 2][h] | (int64_t)a[u / 2][h + 1] << 32;
                    const int64_t xv = (uint32_t)xd[u / 2][t][h] | (int64_t)xd[u / 2][t][h + 1] << 32;
                    p[t] = __builtin_amdgcn_mfma_i32_16x16x32_i8(av, xv, p[t], 0, 0, 0);
                }
            }
            const int grp = b * PER + u;
            const uint2 sc = *reinterpret_cast<const uint2*>(l.scale + ((int64_t)tile * l.groups + grp) * 16 + g4 * 4);
            const float sw[4] = {bf16_lo(sc.x), bf16_hi(sc.x), bf16_lo(sc.y), bf16_hi(sc.y)};
            const float sx = dg.scale[((int64_t)mt * l.groups + grp) * 16 + (lane & 15)];
            if (ZERO) {
                const uint32_t z = *reinterpret_cast<const uint32_t*>(l.zero + ((int64_t)tile * l.groups + grp) * 16 + g4 * 4);
#pragma unroll
                for (int t = 0; t < 3; ++t) {
                    const int s = 16 * dg.sum[(((int64_t)mt * l.groups + grp) * 3 + t) * 16 + (lane & 15)];
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[t][r] -= (int)(int8_t)(z >> (8 * r)) * s;
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float v = fmaf((float)p[2][r], 65536.f, fmaf((float)p[1][r], 256.f, (float)p[0][r]));
                acc[r] = fmaf(v * sx, sw[r], acc[r]);
            }
        }
    }
    const int64_t m = (int64_t)mt * 16 + (lane & 15);
    if (m >= M) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t n = (int64_t)tile * 16 + 4 * g4 + r;
        if (n < l.N) y[m * l.N + n] = accumulate ? y[m * l.N + n] + acc[r] : acc[r];
    }
}

}  // namespace chiron

struct chiron_linear4 {
    chiron::Linear4 L;
    int device = -1;
};

using namespace chiron;

extern "C" {

int32_t chiron_linear4_destroy(chiron_linear4* l) {
    if (!l) return CHIRON_OK;
    if (l->L.w) (void)hipFree(l->L.w);
    if (l->L.scale) (void)hipFree(l->L.scale);
    if (l->L.zero) (void)hipFree(l->L.zero);
    scratch_pool_leave(l->device);
    delete l;
    return CHIRON_OK;
}

int32_t chiron_linear4_create(const void* w4, const void* scales, const void* zeros, int32_t N, int32_t K, int32_t group, void* stream,
                              chiron_linear4** out) {
    if (!out) return fail(CHIRON_ERR_INVALID_ARG, "out is null");
    *out = nullptr;
    if (!w4 || !scales || N < 1 || K < 1) return fail(CHIRON_ERR_INVALID_ARG, "linear4: null weight or scale, or a non-positive size");
    if (group != 32 && group != 64 && group != 128) return fail(CHIRON_ERR_SHAPE, "linear4: group %d must be 32, 64 or 128", group);
    if (K % group != 0) return fail(CHIRON_ERR_SHAPE, "linear4: K=%d must be a multiple of the group %d", K, group);
    if ((uintptr_t)scales & 1) return fail(CHIRON_ERR_INVALID_ARG, "linear4: scales must be 2-byte aligned");
    const int64_t tiles = ((int64_t)N + 15) / 16, kb = ((int64_t)K + 127) / 128;
    if (tiles * kb * 64 / 256 >= 0x7fffffff || kb * 128 > 0x7fffffff) return fail(CHIRON_ERR_SHAPE, "linear4: %d x %d is too large", N, K);
    chiron_linear4* l = new (std::nothrow) chiron_linear4();
    if (!l) return fail(CHIRON_ERR_OOM, "host allocation failed");
    Linear4& L = l->L;
    L.N = N; L.K = K; L.group = group; L.Kpad = (int)(kb * 128); L.groups = L.Kpad / group;
    const int64_t ns = tiles * 16 * L.groups;
    int32_t rc = dev_alloc((void**)&L.w, (size_t)(tiles * kb * 1024));
    if (!rc) rc = dev_alloc((void**)&L.scale, (size_t)ns * 2);
    if (!rc && zeros) rc = dev_alloc((void**)&L.zero, (size_t)ns);
    if (!rc) {
        hipStream_t st = (hipStream_t)stream;
        launch(pack4_kernel, dim3((unsigned)((tiles * kb * 64 + 255) / 256)), dim3(256), st, (const uint8_t*)w4, L);
        launch(pack4_scales_kernel, dim3((unsigned)((ns + 255) / 256)), dim3(256), st, (const uint16_t*)scales, (const uint8_t*)zeros, L);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) rc = fail(CHIRON_ERR_HIP, "linear4: %s", hipGetErrorString(e));
    }
    if (rc) {
        chiron_linear4_destroy(l);
        return rc;
    }
    l->device = scratch_pool_enter();
    *out = l;
    return CHIRON_OK;
}

int32_t chiron_op_linear4(const chiron_linear4* l, const float* x, int32_t M, float* y, int32_t accumulate, void* stream) {
    if (!l) return fail(CHIRON_ERR_INVALID_ARG, "linear is null");
    if (M < 0) return fail(CHIRON_ERR_INVALID_ARG, "M is negative");
    if (M == 0) return CHIRON_OK;
    if (!x || !y) return fail(CHIRON_ERR_INVALID_ARG, "linear4: a pointer is null");
    if (((uintptr_t)x | (uintptr_t)y) & 3) return fail(CHIRON_ERR_INVALID_ARG, "linear4: x or y is misaligned");
    const Linear4& L = l->L;
    if (x < y + (size_t)M * L.N && y < x + (size_t)M * L.K) return fail(CHIRON_ERR_INVALID_ARG, "linear4: x and y overlap");
    const int64_t mt = ((int64_t)M + 15) / 16, kb = L.Kpad / 128;
    if (mt > 65535) return fail(CHIRON_ERR_BATCH_TOO_LARGE, "linear4: %d rows, at most %d", M, 65535 * 16);
    hipStream_t st = (hipStream_t)stream;
    const int64_t digit_bytes = mt * kb * 6 * 1024, scale_bytes = mt * L.groups * 64, sum_bytes = L.zero ? mt * L.groups * 192 : 0;
    void* scratch = nullptr;
    int32_t rc = scratch_alloc(l->device, &scratch, (size_t)(digit_bytes + scale_bytes + sum_bytes), st);
    if (rc) return rc;
    Digits dg;
    dg.d = (uint8_t*)scratch;
    dg.scale = (float*)(dg.d + digit_bytes);
    dg.sum = L.zero ? (int32_t*)(dg.d + digit_bytes + scale_bytes) : nullptr;
    launch(digits_kernel, dim3((unsigned)kb, (unsigned)mt), dim3(64), st, x, M, L, dg);
    const dim3 grid((unsigned)((((int64_t)L.N + 15) / 16 + 3) / 4), (unsigned)mt);
#define CHIRON_L4(G_)                                                                                    \
    do {                                                                                                 \
        if (L.zero) launch(linear4_kernel<G_, true>, grid, dim3(256), st, L, dg, M, y, accumulate);      \
        else launch(linear4_kernel<G_, false>, grid, dim3(256), st, L, dg, M, y, accumulate);            \
    } while (0)
    if (L.group == 128) CHIRON_L4(128);
    else if (L.group == 64) CHIRON_L4(64);
    else CHIRON_L4(32);
#undef CHIRON_L4
    const hipError_t e = hipGetLastError();
    (void)hipFreeAsync(scratch, st);
    if (e != hipSuccess) return fail(CHIRON_ERR_HIP, "linear4: %s", hipGetErrorString(e));
    return CHIRON_OK;
}

}  // extern "C"
