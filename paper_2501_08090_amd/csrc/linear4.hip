// Products of few rows with 4-bit weights: y = x W^T, W[n][k] = (w4 - z) * scale, a scale and a zero point for each row and group of
// 32, 64 or 128 inputs.  gfx950, wave64.
//
// x enters on two ways, of which neither loses what is small beside something large:
//  - few rows (passes of up to 16), where bringing x to the matrix cores costs most, per row and 128 inputs as whole multiples of a power of
//    two, |x| < 2^31, in four signed 8-bit digits: 31 bits of the largest value, so that an input of fp32's own 24 bits loses none of them
//    until it is 2^-7 of that, and one of 2^-10 of it keeps 21.  (Three digits left 13 of those, and did not use the last quarter of the matrix
//    operands' columns.)  A group's digit sums are exact, and are scaled and added over the groups in fp32.  A weight without zero points is
//    16 * (w4 - 8), which is its four bits, the highest inverted when the matrix is laid out, in the upper half of a byte: three
//    instructions for eight weights.  With zero points it is w4 - z: eight bytes, seven instructions.
//  - many rows as two fp16 terms (off by 2^-22 of an input and 2^-39 of the largest of its 128), whose products with w4 - z, exact in fp16,
//    meet in one fp32 sum.
// (Scales multiply sums, not weights: w4 - z times a bf16 scale has 12 bits, one more than fp16.)
//
// Layout: tiles of 16 rows of W and 128 of K, 1 KiB each, a tile's blocks one behind the other: lane l holds row l % 16 and 32 values
// of K in one 16-byte load, two dwords for each step of 64.  Within a step byte j of lane group g is k = 32 * (j / 8) + 8 g + j % 8,
// for W and x alike, so that a group of 32 is what the halves of the operand registers hold.  Scales and zero points lie as
// [tile][block][row][group of the block], so that what a lane needs of a block is one load.
#include <algorithm>
#include <cmath>
#include <new>

#include "draft_ops.h"

namespace chiron {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct Linear4 {
    uint8_t* w = nullptr;       // [N/16][K/128][64 lanes][16 B]
    uint16_t* scale = nullptr;  // [N/16][K/128][16][128/group] bf16
    uint8_t* zero = nullptr;    // the same, 128 - z, or null
    int N = 0, K = 0, group = 0, Kpad = 0;
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
            uint32_t q = 8;  // outside: scale 0, or digits 0
            if (n < l.N && k < l.K) {
                const uint8_t two = w4[n * (l.K / 2) + k / 2];
                q = (k & 1) ? two >> 4 : two & 15;
            }
            v |= (l.zero ? q : q ^ 8) << (i < 4 ? 8 * i + 4 : 8 * (i - 4));  // the first four in the upper halves of the bytes
        }
        out[d] = v;
    }
    *reinterpret_cast<uint4*>(l.w + j * 16) = make_uint4(out[0], out[1], out[2], out[3]);
}

// Zero points up to 64: w4 - z is exact in all that the kernels make of it (64 + z is a whole number of fp16's steps up to there).
// too_large: set where one is larger.
constexpr int kMaxZero = 64;
__global__ __launch_bounds__(256) void pack4_scales_kernel(const uint16_t* __restrict__ scales, const uint8_t* __restrict__ zeros, Linear4 l, uint32_t* too_large) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;  // (tile, block, row, group of the block)
    const int per = 128 / l.group, kb = l.Kpad / 128, live = l.K / l.group;
    const int64_t tb = j / (16 * per), tile = tb / kb;
    if (tile * 16 >= l.N) return;
    const int w = (int)(j % (16 * per));
    const int64_t n = tile * 16 + w / per;
    const int g = (int)(tb % kb) * per + w % per;
    const bool there = n < l.N && g < live;
    l.scale[j] = there ? scales[n * live + g] : 0;
    if (l.zero) {
        const int z = there ? zeros[n * live + g] : 0;
        l.zero[j] = (uint8_t)(128 - min(z, kMaxZero));
        if (z > kMaxZero) *too_large = 1;
    }
}

// ---- pieces that the kernels share -----------------------------------------------------------------------------
// a dword of eight weights as two registers of four signed bytes: what the upper halves of its bytes hold, then the lower ones;
// z4: the lane's row's 128 - z in every byte
template <bool ZERO>
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t z4, int& upper, int& lower) {
    if (ZERO) {  // w4 + (128 - z) stays within a byte; the highest bit inverted makes it w4 - z
        upper = (int)((((w >> 4) & 0x0f0f0f0fu) + z4) ^ 0x80808080u);
        lower = (int)(((w & 0x0f0f0f0fu) + z4) ^ 0x80808080u);
    } else {
        upper = (int)(w & 0xf0f0f0f0u);
        lower = (int)((w << 4) & 0xf0f0f0f0u);
    }
}
// a block's operand of W: two steps of 64
template <int GROUP, bool ZERO>
__device__ __forceinline__ void unpack_block(const uint4& w, uint32_t zbytes, intx4 (&a)[2]) {
    const uint32_t wd[4] = {w.x, w.y, w.z, w.w};
    constexpr int PER = 128 / GROUP;
#pragma unroll
    for (int d = 0; d < 4; ++d) {  // dword d lies in the group d * PER / 4 of the block
        const uint32_t z4 = ZERO ? __builtin_amdgcn_perm(zbytes, zbytes, 0x01010101u * (d * PER / 4)) : 0;
        int u, l;
        unpack8<ZERO>(wd[d], z4, u, l);
        a[d / 2][d % 2 * 2] = u;
        a[d / 2][d % 2 * 2 + 1] = l;
    }
}
template <int GROUP>
__device__ __forceinline__ uint32_t load_zeros(const uint8_t* zero, int64_t tb, int row) {
    constexpr int PER = 128 / GROUP;
    const uint8_t* p = zero + (tb * 16 + row) * PER;
    return PER == 4 ? *reinterpret_cast<const uint32_t*>(p) : PER == 2 ? *reinterpret_cast<const uint16_t*>(p) : *p;
}
// the scales of a block for the accumulator's rows 4g .. 4g+3: PER for each row
template <int GROUP>
struct Scales {
    uint2 v[128 / GROUP];
    __device__ __forceinline__ void load(const uint16_t* scale, int64_t tb, int g4) {
        const uint2* p = reinterpret_cast<const uint2*>(scale + (tb * 16 + g4 * 4) * (128 / GROUP));
#pragma unroll
        for (int i = 0; i < 128 / GROUP; ++i) v[i] = p[i];
    }
    __device__ __forceinline__ float get(int row, int u) const {
        const int i = row * (128 / GROUP) + u;
        const uint32_t w = i % 4 / 2 ? v[i / 4].y : v[i / 4].x;
        return i % 2 ? bf16_hi(w) : bf16_lo(w);
    }
};
// whole-number product of group u of a block
template <int GROUP>
__device__ __forceinline__ intx4 group_product(const intx4 (&a)[2], const intx4 (&x)[2], int u) {
    intx4 p = {0, 0, 0, 0};
    if constexpr (GROUP == 128) {
        p = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[0], x[0], p, 0, 0, 0);
        p = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[1], x[1], p, 0, 0, 0);
    } else if constexpr (GROUP == 64) {
        p = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u], x[u], p, 0, 0, 0);
    } else {
        const int h = (u & 1) * 2;
        const int64_t av = (uint32_t)a[u / 2][h] | (int64_t)a[u / 2][h + 1] << 32;
        const int64_t xv = (uint32_t)x[u / 2][h] | (int64_t)x[u / 2][h + 1] << 32;
        p = __builtin_amdgcn_mfma_i32_16x16x32_i8(av, xv, p, 0, 0, 0);
    }
    return p;
}
// four digits' sums as one value; two of them stay below 2^30 (128 products of at most 128 * 128 each)
__device__ __forceinline__ float join_digits(int p3, int p2, int p1, int p0) { return fmaf((float)((p3 << 8) + p2), 65536.f, (float)((p1 << 8) + p0)); }

// A block's power of two from the bits of its largest magnitude: x * 2^up is below 0.9922 * 2^31, where four signed digits end a little
// higher.  (Below 2^-96 the digits stop at 2^-127.)
__device__ __forceinline__ int exponent_up(uint32_t top) {
    return min(127, 31 - __builtin_amdgcn_frexp_expf(__uint_as_float(top)) - ((top & 0x7fffffu) >= 0x7e0000u));
}
// what the lowest digit counts; without zero points weights are 16 times themselves.  Infinity or NaN in the block: NaN
template <bool ZERO>
__device__ __forceinline__ float block_scale(uint32_t top) {
    return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, -exponent_up(top) - (ZERO ? 0 : 4));
}
// 8 consecutive values of a row as signed 8-bit digits q = 2^24 d3 + 2^16 d2 + 2^8 d1 + d0, highest first, of x * 2^up rounded to a whole
// number (to nearest, ties to even); 0x808080 more carries into the next digit where one is above 127 and leaves the lower three in their
// bytes with the highest bit inverted.
struct Run {
    uint2 digit[4];
};
__device__ __forceinline__ Run digits_of(const float (&v)[8], uint32_t top) {
    const float up = top >= 0x7f800000u ? 0.f : ldexpf(1.f, exponent_up(top));
    Run r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = (uint32_t)(int)rintf(v[4 * h + i] * up) + 0x808080u;
        const uint32_t a = __builtin_amdgcn_perm(q[1], q[0], 0x05010400u), b = __builtin_amdgcn_perm(q[3], q[2], 0x05010400u);  // d0 d0 d1 d1
        const uint32_t c = __builtin_amdgcn_perm(q[1], q[0], 0x07030602u), d = __builtin_amdgcn_perm(q[3], q[2], 0x07030602u);  // d2 d2 d3 d3
        const uint32_t digit[4] = {__builtin_amdgcn_perm(d, c, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x05040100u) ^ 0x80808080u,
                                   __builtin_amdgcn_perm(b, a, 0x07060302u) ^ 0x80808080u, __builtin_amdgcn_perm(b, a, 0x05040100u) ^ 0x80808080u};
#pragma unroll
        for (int t = 0; t < 4; ++t) (h == 0 ? r.digit[t].x : r.digit[t].y) = digit[t];
    }
    return r;
}
// values k .. k+7 of a row of x, zeros behind K (a multiple of 32).  Rows need no more than their type's alignment: a 16-byte load of
// global memory does with 4 bytes, and two ways to load would be a branch around every one of them.
typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void load_run(const float* row, int k, int K, float (&v)[8]) {
    const int at = min(k, K - 8);
    const floatx4_any a = *reinterpret_cast<const floatx4_any*>(row + at), b = *reinterpret_cast<const floatx4_any*>(row + at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = k < K ? a[i] : 0.f;
        v[4 + i] = k < K ? b[i] : 0.f;
    }
}
// the largest magnitude of a run's block of 128 as bits (infinities and NaN come out on top); lanes hold consecutive runs, 16 to a block
__device__ __forceinline__ uint32_t block_top(const float (&v)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)row_move<kRor8>((int)top));
    top = max(top, (uint32_t)row_move<kRor4>((int)top));
    top = max(top, (uint32_t)row_move<kRor2>((int)top));
    return max(top, (uint32_t)row_move<kRor1>((int)top));
}

// ---- few rows --------------------------------------------------------------------------------------------------
// A workgroup converts its slice of x to digits once, in LDS, and then walks tiles of 16 columns; its 8 waves own NB blocks of K each,
// whose x stays in registers, and add their sums through LDS.  With up to 4 rows the four digits of a row take different columns of
// one operand (column = 4 * digit + row), with up to 8 those of two operands (8 * (digit % 2) + row), else four.  A slice of more than 8 NB blocks
// goes in chunks, whose sums wait in LDS (for kFewTiles tiles at most): adding them up in y would put a load behind the weights on their
// way, and what it waits for would be all of them.  The loops hold no branch that depends on a wave: blocks behind the slice's end
// read the last one again and count with 0.  8 rows through 28672 x 4096: 17 us, 3.6 TB/s; one through 4096 x 4096: 5.1.
// Bound by what stands before and beside the stream of weights: the launch, bringing x in (its conversion is a chain of loads, a maximum
// over 16 lanes and LDS) and, with more rows, the scaling of the digits' sums.
// Digits lie in LDS as the operands want them, 16 bytes a lane, column c of lane group g and step k in the place c ^ (4 g + k % 4) of its
// 16: lanes that write consecutive runs of a row then meet in no bank.
constexpr int kFewTiles = 12;
__device__ __forceinline__ int few_slot(int k64, int g, int c) { return g * 16 + (c ^ (g * 4 + (k64 & 3))); }
// ONE: no workgroup has more than one tile, so that there is nothing to read ahead.
template <int GROUP, bool ZERO, int SETS, int NB, bool ONE>
__global__ __launch_bounds__(512, 2) void linear4_few_kernel(Linear4 l, const float* __restrict__ x, int rows, int pass_rows, int slice_blocks, float* __restrict__ y,
                                                             int accumulate) {
    constexpr int PER = 128 / GROUP, ROWS = 4 * SETS;
    // tiles on their way: as many as the registers hold beside x
    constexpr int RING = ONE ? 1 : NB == 4 ? (GROUP == 32 || SETS == 2 ? 2 : 3) : NB == 2 ? (SETS == 4 ? (GROUP == 32 ? 1 : 3) : GROUP == 32 ? 3 : 4) : 6;
    __shared__ uint4 s_dig[NB * 8 * 2 * SETS * 64];
    __shared__ float s_base[NB * 8][ROWS];
    __shared__ __align__(16) float s_red[2][8][256];
    __shared__ float s_acc[kFewTiles][256];
    const int lane = threadIdx.x & 63, col = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kb = l.Kpad / 128, tiles = (l.N + 15) / 16;
    const int out_row = threadIdx.x & 15, out_m = threadIdx.x >> 4;  // what a thread writes of a tile
    const int k0 = blockIdx.y * slice_blocks, k1 = min(kb, k0 + slice_blocks);
    const int m0 = blockIdx.z * pass_rows, M = min(pass_rows, rows - m0);  // this pass's rows
    x += (int64_t)m0 * l.K;
    y += ((int64_t)blockIdx.y * rows + m0) * l.N;
    // what digit a column holds in each set: weight 2^(24 - 8 digit)
    float f[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        const int d = s * (16 / ROWS) + col / ROWS;
        f[s] = d == 0 ? 16777216.f : d == 1 ? 65536.f : d == 2 ? 256.f : 1.f;
    }
    const int step = gridDim.x, home = blockIdx.x;
    int buf = 0;
    for (int c0 = k0; c0 < k1; c0 += NB * 8) {
        const int nbk = min(NB * 8, k1 - c0), b0 = wave * NB;  // blocks of the chunk, this wave's first
        uint4 w[RING][NB];
        Scales<GROUP> sc[RING][NB];
        uint32_t z[RING][NB];
        float old[RING];
        const bool last = c0 + NB * 8 >= k1;
        auto fetch = [&](int tile, int j) {
            old[j] = 0.f;
            if (accumulate && last && out_m < M && tile * 16 + out_row < l.N) old[j] = y[(int64_t)out_m * l.N + tile * 16 + out_row];
            const int64_t tb = (int64_t)tile * kb + c0;
#pragma unroll
            for (int i = 0; i < NB; ++i) w[j][i] = load_stream_16(l.w + ((tb + min(b0 + i, nbk - 1)) * 64 + lane) * 16);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                sc[j][i].load(l.scale, tb + min(b0 + i, nbk - 1), g4);
                if (ZERO) z[j][i] = load_zeros<GROUP>(l.zero, tb + min(b0 + i, nbk - 1), col);
            }
        };
        // All of the chunk's x is asked for before the first weights: loads come back in order, and x, which lies in the L2, need not
        // wait for them.
        constexpr int ROW = NB * 128, U = (ROWS * ROW + 511) / 512;  // runs of 8 in a row of the chunk, runs per thread
        float v[U][8];
#pragma unroll
        for (int i = 0; i < U; ++i) {  // (rows behind the last and blocks behind the chunk: something that is there, not used)
            const int r = i * 512 + threadIdx.x;
            load_run(x + (int64_t)min(r / ROW, M - 1) * l.K, (c0 * 16 + min(r % ROW, nbk * 16 - 1)) * 8, l.K, v[i]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < RING; ++j) fetch(home + j * step < tiles ? home + j * step : home, j);  // on their way while x is converted
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int r = i * 512 + threadIdx.x, m = r / ROW, run = r % ROW;
            const int k64 = run / 8, half = run / 4 % 2, g = run % 4;  // step of 64, half of 32, lane group
            if (m < M && run < nbk * 16) {  // (16 lanes that share a block stay together)
                const uint32_t top = block_top(v[i]);
                const Run d = digits_of(v[i], top);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int set = t / (16 / ROWS), c = t % (16 / ROWS) * ROWS + m;
                    reinterpret_cast<uint2*>(&s_dig[(k64 * SETS + set) * 64 + few_slot(k64, g, c)])[half] = d.digit[t];
                }
                if (run % 16 == 0) s_base[run / 16][m] = block_scale<ZERO>(top);
            }
        }
        lds_barrier();
        intx4 xf[NB][SETS][2];  // (columns of no row hold anything: whole numbers that nobody reads)
        float base[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
#pragma unroll
            for (int s = 0; s < SETS; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) xf[i][s][h] = *reinterpret_cast<const intx4*>(&s_dig[(((b0 + i) * 2 + h) * SETS + s) * 64 + few_slot((b0 + i) * 2 + h, g4, col)]);
            base[i] = b0 + i < nbk ? s_base[b0 + i][col % ROWS] * (SETS == 1 ? f[0] : 1.f) : 0.f;
        }
        auto product = [&](int j) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                intx4 a[2];
                unpack_block<GROUP, ZERO>(w[j][i], z[j][i], a);
                float sum[4];  // of the block's groups, in steps of x
#pragma unroll
                for (int u = 0; u < PER; ++u) {
                    intx4 p[SETS];
#pragma unroll
                    for (int s = 0; s < SETS; ++s) p[s] = group_product<GROUP>(a, xf[i][s], u);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v;
                        if constexpr (SETS == 1) v = (float)p[0][r];
                        else if constexpr (SETS == 2) v = fmaf((float)p[0][r], f[0], (float)p[1][r] * f[1]);
                        else v = join_digits(p[0][r], p[1][r], p[2][r], p[3][r]);
                        sum[r] = u == 0 ? v * sc[j][i].get(r, u) : fmaf(v, sc[j][i].get(r, u), sum[r]);
                    }
                    // one group's sums are done before the next's products begin: the compiler otherwise holds all 32 products, and scratch
                    // memory for what they displace costs 4 us a launch
                    if constexpr (SETS == 4 && GROUP == 32) asm volatile("" : "+v"(sum[0]), "+v"(sum[1]), "+v"(sum[2]), "+v"(sum[3]));
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[r] = fmaf(sum[r], base[i], acc[r]);
            }
            return make_float4(acc[0], acc[1], acc[2], acc[3]);
        };
        auto finish = [&](int t, float was, float4 acc) {
            *reinterpret_cast<float4*>(&s_red[buf][wave][col * 16 + g4 * 4]) = acc;
            lds_barrier();
            if (out_m < M) {
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    v += s_red[buf][w][out_m * 16 + out_row];
                    if (SETS <= 2) v += s_red[buf][w][(out_m + ROWS) * 16 + out_row];
                    if (SETS <= 1) v += s_red[buf][w][(out_m + 2 * ROWS) * 16 + out_row] + s_red[buf][w][(out_m + 3 * ROWS) * 16 + out_row];
                }
                if (k1 - k0 > NB * 8) {  // several chunks: kFewTiles tiles a workgroup at most
                    float& sum = s_acc[(t - home) / step][threadIdx.x];
                    if (c0 > k0) v += sum;
                    if (!last) sum = v;
                }
                if (last && t * 16 + out_row < l.N) y[(int64_t)out_m * l.N + t * 16 + out_row] = v + was;
            }
            buf ^= 1;  // the other half next: this one is read until the next barrier
        };
        // A ring of RING tiles: one's place is filled again as soon as it is multiplied.  (Past the end: the workgroup's first tile, not used.)
        bool more = true;
        for (int t = home; more; t += RING * step) {
#pragma unroll
            for (int j = 0; j < RING; ++j) {
                const int cur = t + j * step, ahead = cur + RING * step;
                if (!more) break;
                const float4 acc = product(j);
                const float was = old[j];
                __builtin_amdgcn_sched_barrier(0);
                if (!ONE) fetch(ahead < tiles ? ahead : home, j);
                __builtin_amdgcn_sched_barrier(0);
                finish(cur, was, acc);
                more = cur + step < tiles;
            }
        }
    }
}

// ---- many rows -------------------------------------------------------------------------------------------------
// x enters as two fp16 terms of x * 2^up, up to 2^15 of a block of 128; a group costs one multiplication and one fused multiply-add for
// each result, where four digits cost six instructions.  64 rows through 8192 x 28672 with groups of 64 and zero points: 80 us, 70 of
// them in this kernel, against 100 and 87 with three digits (17 rows through 28672 x 4096: 29, by passes with four digits 30).  What bounds
// it is the matrix cores and the vector units, which share issue and power: with no products 56 us are left of the 70, with no loads of
// weights or x 60.  The 60 GFLOP run at 0.86 PFLOP/s, a large fp16 product of the library reaches 1.1; the weights take 19 us.
//
// x for the whole launch: terms [rows/16][K/128][4 steps of 32][2][64 lanes][16 B], scales [rows/16][K/128][16] fp32.  A lane's eight
// values of a step lie in the order in which masks take weights out of a dword: (4,6) (0,2) (5,7) (1,3).
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
struct Terms {
    uint8_t* d = nullptr;
    float* scale = nullptr;
};
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
    halfx2 h = {(_Float16)a, (_Float16)b};
    return *reinterpret_cast<uint32_t*>(&h);
}
// a wave per tile of 16 rows and block: a lane holds 8 values of each of the four steps, reads them 128 bytes a row and writes them 1 KiB
// a wave
__global__ __launch_bounds__(256) void terms_kernel(const float* __restrict__ x, int M, Linear4 l, Terms tm) {
    const int kb = l.Kpad / 128, b = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 15, g = lane >> 4;
    const int64_t mt = blockIdx.y, m = mt * 16 + row;  // rows behind M: zeros
    if (b >= kb) return;
    float v[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int step = 0; step < 4; ++step) load_run(x + (m < M ? m : M - 1) * l.K, b * 128 + step * 32 + g * 8, l.K, v[step]);
#pragma unroll
    for (int step = 0; step < 4; ++step)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (m >= M) v[step][i] = 0.f;
            top = max(top, __float_as_uint(v[step][i]) & 0x7fffffffu);
        }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const bool bad = top >= 0x7f800000u;  // infinity or NaN in the block: its scale is NaN
    const int up = min(127, 15 - __builtin_amdgcn_frexp_expf(__uint_as_float(top)));
    const float f = bad ? 0.f : ldexpf(1.f, up);
    uint8_t* out = tm.d + (mt * kb + b) * 8192 + lane * 16;
#pragma unroll
    for (int step = 0; step < 4; ++step) {
        float hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = v[step][i] * f;
            hi[i] = (float)(_Float16)s;
            lo[i] = s - hi[i];
        }
        *reinterpret_cast<uint4*>(out + step * 2048) = make_uint4(pack_half(hi[4], hi[6]), pack_half(hi[0], hi[2]), pack_half(hi[5], hi[7]), pack_half(hi[1], hi[3]));
        *reinterpret_cast<uint4*>(out + step * 2048 + 1024) = make_uint4(pack_half(lo[4], lo[6]), pack_half(lo[0], lo[2]), pack_half(lo[5], lo[7]), pack_half(lo[1], lo[3]));
    }
    if (g == 0) tm.scale[(mt * kb + b) * 16 + row] = bad ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, -up);
}

// Eight weights of a dword as fp16, nine instructions: a mask and the bits of 1024 make 1024 + w4 of the lower four bits of a byte and
// 1024 + 16 w4 of the upper four; then minus 1024 + z, or over 16 and minus 64 + z, exactly.  (Without zero points the highest of the
// four bits lies inverted.)
struct Offsets {
    halfx2 low, high;  // -(1024 + z), -(64 + z)
};
__device__ __forceinline__ halfx2 as_half(uint32_t w) { return *reinterpret_cast<halfx2*>(&w); }
template <bool ZERO>
__device__ __forceinline__ halfx8 unpack_half(uint32_t w, const Offsets& o, uint32_t bits) {
    if (!ZERO) w ^= 0x88888888u;
    const uint32_t v = w >> 8;
    const halfx2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const halfx2 r0 = as_half((w & 0x000f000fu) | bits) + o.low, r2 = as_half((v & 0x000f000fu) | bits) + o.low;
    const halfx2 r1 = __builtin_elementwise_fma(as_half((w & 0x00f000f0u) | bits), sixteenth, o.high);
    const halfx2 r3 = __builtin_elementwise_fma(as_half((v & 0x00f000f0u) | bits), sixteenth, o.high);
    return halfx8{r0[0], r0[1], r1[0], r1[1], r2[0], r2[1], r3[0], r3[1]};
}

// A workgroup of 8 waves owns 256 columns, MT tiles of 16 rows and a slice of K; slices go to `part` and are added by the caller's next
// launch.  Terms and scales pass through LDS block by block.  A wave owns 64 columns and one half of every block, so that all of x is
// read from LDS four times and no weight is unpacked twice; the halves are joined at the end.
//
// A block goes in 2 MT phases, the products of a row tile with two of the wave's column tiles.  The waves go through a block together, so
// what is to run beside the matrix cores has to come from the same wave: beside a phase's products run the scaling of the last phase's
// sums, the reads of the next row tile's operands, in the first phase the unpacking of column tiles 2 and 3, and in the last, where 0 and
// 1 have done their part, that of the next block's 0 and 1.  Weights are asked for again as soon as they are unpacked.  One barrier a
// block: behind it the next block's x is there, and this one's is no longer read.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// 2 GiB from p on, for loads with an offset of the lane and one of the wave; every offset stays inside what p points to
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00027000);
}
template <int GROUP, bool ZERO, int MT>
__global__ __launch_bounds__(512, 2) void linear4_kernel(Linear4 l, Terms tm, int M, int slice_blocks, float* __restrict__ out, int add) {
    constexpr int PER = 128 / GROUP, PERW = PER == 4 ? 2 : 1, NS = MT * 16;  // groups in a block, in a wave's half of it
    __shared__ u32x4 s_x[2][MT * 512];
    __shared__ float s_scale[2][NS];
    const int lane = threadIdx.x & 63, col = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = wave & 1, pair = wave >> 1;
    const int kb = l.Kpad / 128, tiles = (l.N + 15) / 16;
    const int b0 = blockIdx.y * slice_blocks, b1 = min(kb, b0 + slice_blocks), mt0 = blockIdx.z * MT;
    const int tile0 = (blockIdx.x * 4 + pair) * 4;
    floatx4 acc[4][MT];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = floatx4{0.f, 0.f, 0.f, 0.f};
    // what a column tile needs of a block, as it comes from memory
    struct Raw {
        u32x2 w;
        uint32_t z, s[PERW == 2 ? 4 : PER == 2 ? 4 : 2];
    };
    Raw raw[4];
    // the wave's column tiles: offsets of a lane, and of a tile (behind the last: the last)
    int tile_at[4];
    const int first = min(tile0, tiles - 1);
#pragma unroll
    for (int n = 0; n < 4; ++n) tile_at[n] = (min(tile0 + n, tiles - 1) - first) * kb;
    const auto w_rsrc = resource(l.w + (int64_t)first * kb * 1024), s_rsrc = resource(l.scale + (int64_t)first * kb * 16 * PER),
               z_rsrc = resource(l.zero + (int64_t)first * kb * 16 * PER);
    const int w_lane = lane * 16 + half * 8, s_lane = g4 * 8 * PER + (PER == 4 ? half * 4 : 0), z_lane = col * PER + (PER == 4 ? half * 2 : PER == 2 ? half : 0);
    auto load_w = [&](Raw& r, int n, int b) __attribute__((always_inline)) {
        const int t = tile_at[n] + b;
        r.w = __builtin_amdgcn_raw_buffer_load_b64(w_rsrc, w_lane, t * 1024, 0);
        if constexpr (PER == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) r.s[i] = __builtin_amdgcn_raw_buffer_load_b32(s_rsrc, s_lane, t * 128 + i * 8, 0);
        } else if constexpr (PER == 2) {
            const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(s_rsrc, s_lane, t * 64, 0);
            r.s[0] = v.x; r.s[1] = v.y; r.s[2] = v.z; r.s[3] = v.w;
        } else {
            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(s_rsrc, s_lane, t * 32, 0);
            r.s[0] = v.x; r.s[1] = v.y;
        }
        if (ZERO) {
            if constexpr (PER == 4) r.z = __builtin_amdgcn_raw_buffer_load_b16(z_rsrc, z_lane, t * 64, 0);
            else r.z = __builtin_amdgcn_raw_buffer_load_b8(z_rsrc, z_lane, t * 16 * PER, 0);
        }
    };
    uint32_t bits = 0x64006400u;
    asm volatile("" : "+v"(bits));
    halfx8 a[4][2];
    float sc[4][PERW][4];
    auto unpack = [&](int n) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const uint32_t z = ZERO ? (PERW == 2 ? (raw[n].z >> (8 * d)) & 255u : raw[n].z & 255u) : 120u;  // 128 minus the zero point
            const Offsets o = {as_half(0xe480e480u - z * 0x10001u), as_half(0xdc00dc00u - z * 0x100010u)};
            a[n][d] = unpack_half<ZERO>(d ? raw[n].w.y : raw[n].w.x, o, bits);
            asm volatile("" : "+v"(a[n][d]));
        }
    };
    auto scales = [&](int n) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if constexpr (PER == 4) {
                sc[n][0][r] = bf16_lo(raw[n].s[r]);
                sc[n][1][r] = bf16_hi(raw[n].s[r]);
            } else if constexpr (PER == 2) {
                sc[n][0][r] = __uint_as_float(__builtin_amdgcn_perm(raw[n].s[r], raw[n].s[r], half ? 0x03020c0cu : 0x01000c0cu));
            } else {
                sc[n][0][r] = r % 2 ? bf16_hi(raw[n].s[r / 2]) : bf16_lo(raw[n].s[r / 2]);
            }
            asm volatile("" : "+v"(sc[n][0][r]));
            if constexpr (PERW == 2) asm volatile("" : "+v"(sc[n][1][r]));
        }
    };
    // x: of the MT row tiles, 8 KiB each, a piece of 16 bytes a thread and tile; their scales.  (The compiler's own vectors: HIP's are
    // copied through scratch memory on their way to LDS.)
    const int tid = threadIdx.x, js = min(tid, NS - 1);
    const auto x_rsrc = resource(tm.d + (int64_t)mt0 * kb * 8192), xs_rsrc = resource(tm.scale + (int64_t)mt0 * kb * 16);
    const int x_lane = tid * 16, xs_lane = (js / 16 * kb * 16 + js % 16) * 4;
    u32x4 x0, x1, x2, x3;
    float xsv;
    auto load_x = [&](int b) __attribute__((always_inline)) {
        x0 = __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, x_lane, b * 8192, 0);
        x1 = __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, x_lane, (kb + b) * 8192, 0);
        if (MT > 2) x2 = __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, x_lane, (2 * kb + b) * 8192, 0);
        if (MT > 3) x3 = __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, x_lane, (3 * kb + b) * 8192, 0);
        xsv = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(xs_rsrc, xs_lane, b * 64, 0));
    };
    auto store_x = [&](int buf) __attribute__((always_inline)) {
        s_x[buf][tid] = x0;
        s_x[buf][512 + tid] = x1;
        if (MT > 2) s_x[buf][1024 + tid] = x2;
        if (MT > 3) s_x[buf][1536 + tid] = x3;
        if (tid < NS) s_scale[buf][tid] = xsv;
    };
    static_assert(MT >= 2 && MT <= 4, "two to four row tiles");
    halfx8 f[2][4];
    float sx[2];
    auto read = [&](int buf, int m, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[to][i] = *reinterpret_cast<const halfx8*>(&s_x[buf][m * 512 + half * 256 + i * 64 + lane]);
        sx[to] = s_scale[buf][m * 16 + col];
    };
    load_x(b0);
#pragma unroll
    for (int n = 0; n < 4; ++n) load_w(raw[n], n, b0);
    store_x(0);
    load_x(min(b0 + 1, b1 - 1));
    unpack(0);
    unpack(1);
    scales(0);
    scales(1);
    load_w(raw[0], 0, min(b0 + 1, b1 - 1));
    load_w(raw[1], 1, min(b0 + 1, b1 - 1));
    lds_barrier();
    read(0, 0, 0);
    int buf = 0;
    for (int b = b0; b < b1; ++b, buf ^= 1) {
        const int b_1 = min(b + 1, b1 - 1), b_2 = min(b + 2, b1 - 1);  // (behind the slice: the last block once more, not used)
        floatx4 p[2][2][PERW];
        float was = 0.f;
#pragma unroll
        for (int ph = 0; ph <= 2 * MT; ++ph) {
            const int m = ph / 2, n0 = ph % 2 * 2, to = ph & 1;
            if (ph < 2 * MT) {
                if (ph % 2 == 0 && m + 1 < MT) read(buf, m + 1, (m + 1) & 1);
                if (ph == 2 * MT - 3) {
                    store_x(buf ^ 1);
                    load_x(b_2);
                }
                if (ph == 2 * MT - 2) lds_barrier();
                if (ph == 2 * MT - 1) read(buf ^ 1, 0, MT & 1);
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int u = 0; u < PERW; ++u) p[to][n][u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int n = 0; n < 2; ++n)
                        p[to][n][i / 2 * (PERW - 1)] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[n0 + n][i / 2], f[m & 1][i], p[to][n][i / 2 * (PERW - 1)], 0, 0, 0);
            }
            if (ph > 0) {  // the last phase's sums
                const int q = ph - 1, pm = q / 2, pn = q % 2 * 2;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float t = p[q & 1][n][0][r] * sc[pn + n][0][r];
                        if constexpr (PERW == 2) t = fmaf(p[q & 1][n][1][r], sc[pn + n][1][r], t);
                        acc[pn + n][pm][r] = fmaf(t, q % 2 ? was : sx[pm & 1], acc[pn + n][pm][r]);
                    }
                    asm volatile("" : "+v"(acc[pn + n][pm]));
                }
            }
            if (ph % 2 == 0 && m < MT) was = sx[m & 1];
            if (ph == 0) {
                unpack(2);
                unpack(3);
                scales(2);
                scales(3);
            }
            if (ph == 2 * MT - 1) {
                unpack(0);
                unpack(1);
            }
            if (ph < 2 * MT) {
                // a product, then a few of the vector instructions, and so on
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (ph == 0 || ph == 2 * MT - 1) __builtin_amdgcn_sched_group_barrier(0x002, 9, 0);
                    else __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (ph == 0) {
                load_w(raw[2], 2, b_1);
                load_w(raw[3], 3, b_1);
            }
        }
        scales(0);
        scales(1);
        __builtin_amdgcn_sched_barrier(0);
        load_w(raw[0], 0, b_2);
        load_w(raw[1], 1, b_2);
        if (MT & 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[0][i] = f[1][i];
            sx[0] = sx[1];
        }
    }
    // The halves are joined, and rows written 1 KiB at a time, through LDS: [row][64 pieces of 4 columns], piece c in the place c ^ row % 16
    // (lanes that hold 16 rows of a piece then meet in no bank).
    lds_barrier();
    floatx4* sum = reinterpret_cast<floatx4*>(&s_x[0][0]);
    auto place = [&](int n, int m) { return (m * 16 + col) * 64 + ((pair * 16 + n * 4 + g4) ^ col); };
    if (half)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) sum[place(n, m)] = acc[n][m];
    lds_barrier();
    if (!half)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) sum[place(n, m)] += acc[n][m];
    lds_barrier();
    float* dst = out + (int64_t)blockIdx.y * M * l.N;
    const int64_t c = (int64_t)blockIdx.x * 256 + lane * 4;
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
        const int r = i * 8 + wave;
        const int64_t row = (int64_t)mt0 * 16 + r;
        if (row >= M || c >= l.N) continue;
        floatx4 v = sum[r * 64 + (lane ^ (r & 15))];
        float* q = dst + row * l.N + c;
        if (c + 4 <= l.N) {
            if (add) v += *reinterpret_cast<const floatx4_any*>(q);
            *reinterpret_cast<floatx4_any*>(q) = v;
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (c + j < l.N) q[j] = add ? q[j] + v[j] : v[j];
        }
    }
}

// How a call of M rows runs: by passes of the few-row kernel, or by tiles of nearly the same height of up to 64 rows, side by side in one
// launch (100 rows through 4096 x 4096: 25.5 us, one behind the other 35.6), K sliced until the chip has a workgroup of 256 columns
// for every CU or further slices cost more than they save.
struct Plan4 {
    int passes = 0, pass_rows = 0, sets = 0, nb = 0, wgs = 0;  // few rows: operands, blocks per wave and chunk, workgroups per slice and pass
    int mt = 0, row_tiles = 0;           // more: row tiles of a workgroup, of all
    int slices = 1, slice_blocks = 0;
    int64_t term_bytes = 0, scale_bytes = 0, part_bytes = 0;
    int64_t bytes() const { return term_bytes + scale_bytes + part_bytes; }
};
static Plan4 plan_linear4(const Linear4& l, int64_t M) {
    Plan4 p;
    const int64_t kb = l.Kpad / 128;
    // More than 16 rows by passes of up to 16 too, as long as all passes' weights stay within 2^27, 1.25 * 2^26 or 2^26 (groups of 128, 64 or
    // 32): one launch, or two, for the tiles' three, but every pass unpacks the weights again, and the smaller the groups, the more of
    // the time goes by results and groups.  us passes / tiles, groups of 128: 64 rows through 4096 x 4096 15.7 / 23.3, 8192 x 4096 (2^27) 22.9 /
    // 26.8, 14336 x 4096 32.7 / 29.6; 32 rows through 4096 x 14336 (1.75 * 2^26) 23.1 / 21.7, 14336 x 4096 21.3 / 21.1; groups of 64 with zero
    // points: 64 rows through 4096 x 4096 (2^26) 19.0 / 24.0, 48 through 5120 x 5120 (1.17 * 2^26) 28.3 / 22.7 and 8192 x 4096 (1.5 * 2^26) 25.3 / 23.8;
    // groups of 32: 64 rows through 2048 x 4096 (2^25) 14.9 / 21.9 and 4096 x 4096 (2^26) 21.2 / 25.1, 32 through 8192 x 4096 (2^26) 21.3 / 20.6, 48
    // through 5120 x 5120 (1.17 * 2^26) 33.3 / 23.7.
    const int64_t passes = (M + 15) / 16, limit = (l.group == 128 ? 8 : l.group == 64 ? 5 : 4) * ((int64_t)1 << 24);
    if (passes == 1 || passes * l.N * kb * 128 <= limit) {
        p.passes = (int)passes;
        p.pass_rows = (int)((M + p.passes - 1) / p.passes);
        p.sets = p.pass_rows <= 4 ? 1 : p.pass_rows <= 8 ? 2 : 4;
        const int64_t most = p.sets == 4 || (p.sets == 2 && l.group == 32) ? 2 : 4;  // what LDS and registers hold
        const int64_t tiles = ((int64_t)l.N + 15) / 16, all = tiles * p.passes;
        // Slices of at most 32 blocks up to 4 rows, of 16 with more, whose x takes a workgroup longer than a second launch and the slices'
        // traffic; 32 too with up to 8 rows where that is all of K and there are tiles for every CU; and of 8, where the chip is not full
        // otherwise.  us with 1 / 2 / 4 / 8 / 16 slices: 1 row through 8192 x 28672 41 / 35 / 29 / 25 / 29, 8 rows through 8192 x 8192
        // 19 / 16 / 13.5 / 15.6 / 25 and through 28672 x 4096 16.8 / 17.5 / 23 / 38 / 67, 16 rows through 1024 x 4096 11.7 / 9.3 / 6.9 /
        // 8.5 / 10.1.
        const bool whole = p.sets == 1 || (p.sets == 2 && kb <= 32 && all >= kNumCU);
        static_assert(kNumCU % 16 == 0, "a slice's share of the CUs is a whole number");
        while (p.slices < 16 && (kb + p.slices - 1) / p.slices > (whole ? 32 : 16)) p.slices *= 2;
        if (!whole && p.slices < 16 && all * p.slices <= 2 * kNumCU && kb / (2 * p.slices) >= 8) p.slices *= 2;
        p.slice_blocks = (int)((kb + p.slices - 1) / p.slices);
        p.slices = (int)((kb + p.slice_blocks - 1) / p.slice_blocks);
        const int64_t chunks = (p.slice_blocks + 8 * most - 1) / (8 * most), need = (p.slice_blocks + 8 * chunks - 1) / (8 * chunks);
        p.nb = need <= 1 ? 1 : need <= 2 ? 2 : 4;
        const int64_t room = std::max<int64_t>(1, kNumCU / (p.slices * p.passes));
        int64_t rounds = (tiles + room - 1) / room;
        if (p.slice_blocks > 8 * p.nb) rounds = std::min<int64_t>(rounds, kFewTiles);
        p.wgs = (int)((tiles + rounds - 1) / rounds);
    } else {
        const int64_t groups = ((int64_t)l.N + 255) / 256;
        const int64_t high = (M + 63) / 64, want = std::max<int64_t>(1, kNumCU / (groups * high));
        p.mt = (int)((passes + high - 1) / high);
        p.row_tiles = (int)(high * p.mt);
        // a block takes a workgroup 1.3 us, a slice's sums to memory and back M N 8 bytes at 4 TB/s: the least of kb 1.3 / s + s M N 2e-6.
        // us with 2 / 4 / 8 / 16 slices, 64 rows: 8192 x 8192 65 / 41 / 31.7 / 41, 14336 x 4096 40 / 30 / 37 / 52, 4096 x 14336 104 / 59 / 37.5 / 30.
        const int64_t least = (int64_t)std::sqrt(6.5e5 * (double)kb / ((double)M * (double)l.N));
        const int64_t slices = std::max<int64_t>(1, std::min(std::min(want, least), kb));
        p.slice_blocks = (int)((kb + slices - 1) / slices);
        p.slices = (int)((kb + p.slice_blocks - 1) / p.slice_blocks);
        p.term_bytes = p.row_tiles * kb * 8192;
        p.scale_bytes = p.row_tiles * kb * 64;
    }
    if (p.slices > 1) p.part_bytes = p.slices * M * l.N * 4;
    return p;
}

template <int GROUP, bool ZERO>
static void launch_linear4(const Linear4& l, const float* x, int M, float* y, int accumulate, const Plan4& p, void* work, hipStream_t st) {
    float* part = (float*)((char*)work + p.term_bytes + p.scale_bytes);
    float* out = p.slices > 1 ? part : y;
    const int add = p.slices > 1 ? 0 : accumulate;
    if (p.passes) {
        const dim3 grid(p.wgs, p.slices, p.passes);
        const bool one = p.wgs == (l.N + 15) / 16;
#define CHIRON_FEW(SETS_, NB_)                                                                                                                        \
    do {                                                                                                                                              \
        if (one) launch(linear4_few_kernel<GROUP, ZERO, SETS_, NB_, true>, grid, dim3(512), st, l, x, M, p.pass_rows, p.slice_blocks, out, add);              \
        else launch(linear4_few_kernel<GROUP, ZERO, SETS_, NB_, false>, grid, dim3(512), st, l, x, M, p.pass_rows, p.slice_blocks, out, add);                 \
    } while (0)
        if (p.sets == 1) {
            if (p.nb == 1) CHIRON_FEW(1, 1);
            else if (p.nb == 2) CHIRON_FEW(1, 2);
            else CHIRON_FEW(1, 4);
        } else if (p.sets == 2) {
            if (p.nb == 1) CHIRON_FEW(2, 1);
            else if (p.nb == 2 || GROUP == 32) CHIRON_FEW(2, 2);
            else if constexpr (GROUP != 32) CHIRON_FEW(2, 4);
        } else {
            if (p.nb == 1) CHIRON_FEW(4, 1);
            else CHIRON_FEW(4, 2);
        }
#undef CHIRON_FEW
        return;
    }
    Terms tm;
    tm.d = (uint8_t*)work;
    tm.scale = (float*)(tm.d + p.term_bytes);
    launch(terms_kernel, dim3((l.Kpad / 128 + 3) / 4, p.row_tiles), dim3(256), st, x, M, l, tm);
    const dim3 grid((l.N + 255) / 256, p.slices, p.row_tiles / p.mt);
    if (p.mt == 4) launch(linear4_kernel<GROUP, ZERO, 4>, grid, dim3(512), st, l, tm, M, p.slice_blocks, out, add);
    else if (p.mt == 3) launch(linear4_kernel<GROUP, ZERO, 3>, grid, dim3(512), st, l, tm, M, p.slice_blocks, out, add);
    else launch(linear4_kernel<GROUP, ZERO, 2>, grid, dim3(512), st, l, tm, M, p.slice_blocks, out, add);
}

}  // namespace chiron

struct chiron_linear4 {
    chiron::Linear4 L;
};

using namespace chiron;

extern "C" {

int32_t chiron_linear4_destroy(chiron_linear4* l) {
    if (!l) return CHIRON_OK;
    if (l->L.w) (void)hipFree(l->L.w);
    if (l->L.scale) (void)hipFree(l->L.scale);
    if (l->L.zero) (void)hipFree(l->L.zero);
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
    if (tiles * kb * 64 / 256 >= 0x7fffffff || kb >= 65536) return fail(CHIRON_ERR_SHAPE, "linear4: %d x %d is too large", N, K);
    chiron_linear4* l = new (std::nothrow) chiron_linear4();
    if (!l) return fail(CHIRON_ERR_OOM, "host allocation failed");
    Linear4& L = l->L;
    L.N = N; L.K = K; L.group = group; L.Kpad = (int)(kb * 128);
    const int64_t ns = tiles * 16 * (L.Kpad / group);
    int32_t rc = dev_alloc((void**)&L.w, (size_t)(tiles * kb * 1024));
    if (!rc) rc = dev_alloc((void**)&L.scale, (size_t)ns * 2);
    if (!rc && zeros) rc = dev_alloc((void**)&L.zero, (size_t)ns + 4);  // behind them a word: one is too large
    if (!rc) {
        hipStream_t st = (hipStream_t)stream;
        uint32_t* flag = zeros ? (uint32_t*)(L.zero + ns) : nullptr;
        uint32_t too_large = 0;
        hipError_t e = zeros ? hipMemsetAsync(flag, 0, 4, st) : hipSuccess;
        launch(pack4_kernel, dim3((unsigned)((tiles * kb * 64 + 255) / 256)), dim3(256), st, (const uint8_t*)w4, L);
        launch(pack4_scales_kernel, dim3((unsigned)((ns + 255) / 256)), dim3(256), st, (const uint16_t*)scales, (const uint8_t*)zeros, L, flag);
        if (e == hipSuccess) e = hipGetLastError();
        if (e == hipSuccess && zeros) e = hipMemcpyAsync(&too_large, flag, 4, hipMemcpyDeviceToHost, st);
        if (e == hipSuccess && zeros) e = hipStreamSynchronize(st);
        if (e != hipSuccess) rc = fail(CHIRON_ERR_HIP, "linear4: %s", hipGetErrorString(e));
        else if (too_large) rc = fail(CHIRON_ERR_INVALID_ARG, "linear4: a zero point is above %d", kMaxZero);
    }
    if (rc) {
        chiron_linear4_destroy(l);
        return rc;
    }
    *out = l;
    return CHIRON_OK;
}

int64_t chiron_linear4_workspace_bytes(const chiron_linear4* l, int32_t M) {
    return l && M > 0 ? plan_linear4(l->L, M).bytes() : 0;
}

int32_t chiron_op_linear4(const chiron_linear4* l, const float* x, int32_t M, float* y, int32_t accumulate, void* workspace, void* stream) {
    if (!l) return fail(CHIRON_ERR_INVALID_ARG, "linear is null");
    if (M < 0) return fail(CHIRON_ERR_INVALID_ARG, "M is negative");
    if (M == 0) return CHIRON_OK;
    if (!x || !y) return fail(CHIRON_ERR_INVALID_ARG, "linear4: a pointer is null");
    if (((uintptr_t)x | (uintptr_t)y) & 3) return fail(CHIRON_ERR_INVALID_ARG, "linear4: x or y is misaligned");
    const Linear4& L = l->L;
    if (x < y + (size_t)M * L.N && y < x + (size_t)M * L.K) return fail(CHIRON_ERR_INVALID_ARG, "linear4: x and y overlap");
    if (M > 65535) return fail(CHIRON_ERR_BATCH_TOO_LARGE, "linear4: %d rows, at most 65535", M);
    const Plan4 p = plan_linear4(L, M);
    if (p.bytes() && !workspace) return fail(CHIRON_ERR_INVALID_ARG, "linear4: %d rows need a workspace", M);
    if ((uintptr_t)workspace & 15) return fail(CHIRON_ERR_INVALID_ARG, "linear4: the workspace must be 16-byte aligned");
    hipStream_t st = (hipStream_t)stream;
#define CHIRON_L4(G_)                                                                      \
    do {                                                                                   \
        if (L.zero) launch_linear4<G_, true>(L, x, M, y, accumulate, p, workspace, st);    \
        else launch_linear4<G_, false>(L, x, M, y, accumulate, p, workspace, st);          \
    } while (0)
    if (L.group == 128) CHIRON_L4(128);
    else if (L.group == 64) CHIRON_L4(64);
    else CHIRON_L4(32);
#undef CHIRON_L4
    CHIRON_HIP(hipGetLastError());
    if (p.slices > 1) return launch_reduce_partials((const float*)((char*)workspace + p.term_bytes + p.scale_bytes), p.slices, (int64_t)M * L.N, y, accumulate, st);
    return CHIRON_OK;
}

}  // extern "C"
