// Products of few rows with 4-bit weights: y = x W^T, W[n][k] = (w4 - z) * scale, a scale and a zero point for each row and group of
// 32, 64 or 128 inputs.  gfx950, wave64.
//
// Within a group the product is whole-number arithmetic on the 8-bit matrix cores.  x enters, per row and 128 inputs, as whole
// multiples of a power of two, |x| <= 2^22, in three signed 8-bit digits; a group's digit sums are exact, and are scaled and added
// over the groups in fp32.  (The digits take the place of the two or three bf16 terms that the other projections split x into: whole numbers need no
// correction for how a weight is unpacked, and the 8-bit matrix cores run at twice the rate.)  A weight without zero points enters as
// 16 * (w4 - 8), which is its four bits, the highest inverted when the matrix is laid out, in the upper half of a byte: three
// instructions for eight weights.  With zero points it enters as w4 - z: eight bytes, seven instructions.
//
// Layout: tiles of 16 rows of W and 128 of K, 1 KiB each, a tile's blocks one behind the other: lane l holds row l % 16 and 32 values
// of K in one 16-byte load, two dwords for each step of 64.  Within a step byte j of lane group g is k = 32 * (j / 8) + 8 g + j % 8,
// for W and x alike, so that a group of 32 is what the halves of the operand registers hold.  Scales and zero points lie as
// [tile][block][row][group of the block], so that what a lane needs of a block is one load.
#include <algorithm>
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

__global__ __launch_bounds__(256) void pack4_scales_kernel(const uint16_t* __restrict__ scales, const uint8_t* __restrict__ zeros, Linear4 l) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;  // (tile, block, row, group of the block)
    const int per = 128 / l.group, kb = l.Kpad / 128, live = l.K / l.group;
    const int64_t tb = j / (16 * per), tile = tb / kb;
    if (tile * 16 >= l.N) return;
    const int w = (int)(j % (16 * per));
    const int64_t n = tile * 16 + w / per;
    const int g = (int)(tb % kb) * per + w % per;
    const bool there = n < l.N && g < live;
    l.scale[j] = there ? scales[n * live + g] : 0;
    if (l.zero) l.zero[j] = there ? (uint8_t)(128 - (zeros[n * live + g] & 15)) : 128;
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
// three digits' sums as one value; the lower two stay below 2^30 (128 products of at most 128 * 128 each)
__device__ __forceinline__ float join_digits(int p2, int p1, int p0) { return fmaf((float)p2, 65536.f, (float)((p1 << 8) + p0)); }

// A block's power of two from the bits of its largest magnitude: x * 2^up is at most 2^22.  (Below 2^-105 the digits stop at 2^-127.)
__device__ __forceinline__ int exponent_up(uint32_t top) { return min(127, 22 - __builtin_amdgcn_frexp_expf(__uint_as_float(top))); }
// what the lowest digit counts; without zero points weights are 16 times themselves.  Infinity or NaN in the block: NaN
template <bool ZERO>
__device__ __forceinline__ float block_scale(uint32_t top) {
    return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, -exponent_up(top) - (ZERO ? 0 : 4));
}
// 8 consecutive values of a row as signed 8-bit digits q = 65536 d2 + 256 d1 + d0, highest first.  Adding 1.5 * 2^23 rounds x * 2^up to
// a whole number (to nearest, ties to even) and leaves it in the low bits; 0x8080 more carries into the next digit where one is above
// 127 and leaves d0 and d1 in their bytes with the highest bit inverted.
struct Run {
    uint2 digit[3];
};
__device__ __forceinline__ Run digits_of(const float (&v)[8], uint32_t top) {
    const float up = top >= 0x7f800000u ? 0.f : ldexpf(1.f, exponent_up(top));
    Run r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = __float_as_uint(fmaf(v[4 * h + i], up, 12582912.f)) - 0x4b400000u + 0x8080u;
        const uint32_t a = __builtin_amdgcn_perm(q[1], q[0], 0x05010400u), b = __builtin_amdgcn_perm(q[3], q[2], 0x05010400u);  // d0 d0 d1 d1
        const uint32_t c = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0602u), d = __builtin_amdgcn_perm(q[3], q[2], 0x0c0c0602u);  // d2 d2
        const uint32_t d0 = __builtin_amdgcn_perm(b, a, 0x05040100u) ^ 0x80808080u, d1 = __builtin_amdgcn_perm(b, a, 0x07060302u) ^ 0x80808080u;
        const uint32_t d2 = __builtin_amdgcn_perm(d, c, 0x05040100u);
        if (h == 0) {
            r.digit[0].x = d2; r.digit[1].x = d1; r.digit[2].x = d0;
        } else {
            r.digit[0].y = d2; r.digit[1].y = d1; r.digit[2].y = d0;
        }
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
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    return top;
}

// ---- up to 16 rows ---------------------------------------------------------------------------------------------
// A workgroup converts its slice of x to digits once, in LDS, and then walks tiles of 16 columns; its 8 waves own NB blocks of K each,
// whose x stays in registers, and add their sums through LDS.  With up to 4 rows the three digits of a row take different columns of
// one operand (column = 4 * digit + row), with up to 8 two operands (8 * digit + row), else three.  A slice of more than 8 NB blocks
// goes in chunks, whose sums wait in LDS (for kFewTiles tiles at most): adding them up in y would put a load behind the weights on their
// way, and what it waits for would be all of them.  The loops hold no branch that depends on a wave: blocks behind the slice's end
// read the last one again and count with 0.
// Digits lie in LDS as the operands want them, 16 bytes a lane, column c of lane group g and step k in the place c ^ (4 g + k % 4) of its
// 16: lanes that write consecutive runs of a row then meet in no bank.
constexpr int kFewTiles = 12;
__device__ __forceinline__ int few_slot(int k64, int g, int c) { return g * 16 + (c ^ (g * 4 + (k64 & 3))); }
// ONE: no workgroup has more than one tile, so that there is nothing to read ahead.
template <int GROUP, bool ZERO, int SETS, int NB, bool ONE>
__global__ __launch_bounds__(512, 2) void linear4_few_kernel(Linear4 l, const float* __restrict__ x, int M, int slice_blocks, float* __restrict__ y,
                                                             int accumulate) {
    constexpr int PER = 128 / GROUP, ROWS = SETS == 1 ? 4 : SETS == 2 ? 8 : 16;
    // tiles on their way: as many as the registers hold beside x
    constexpr int RING = ONE ? 1 : NB == 8 ? 2 : NB == 4 ? (GROUP == 32 || SETS == 2 ? 2 : 3) : NB == 2 ? (SETS == 3 ? (GROUP == 32 ? 1 : 3) : GROUP == 32 ? 3 : 4) : 6;
    __shared__ uint4 s_dig[NB * 8 * 2 * SETS * 64];
    __shared__ float s_base[NB * 8][ROWS];
    __shared__ __align__(16) float s_red[2][8][256];
    __shared__ float s_acc[kFewTiles][256];
    const int lane = threadIdx.x & 63, col = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kb = l.Kpad / 128, tiles = (l.N + 15) / 16;
    const int out_row = threadIdx.x & 15, out_m = threadIdx.x >> 4;  // what a thread writes of a tile
    const int k0 = blockIdx.y * slice_blocks, k1 = min(kb, k0 + slice_blocks);
    y += (int64_t)blockIdx.y * M * l.N;
    // what digit a column holds in each set: weight 2^(16 - 8 digit), none behind the third
    float f[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        const int d = s * (16 / ROWS) + col / ROWS;
        f[s] = d == 0 ? 65536.f : d == 1 ? 256.f : d == 2 ? 1.f : 0.f;
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
        // wait for them (8 rows through 28672 x 4096: %s us).
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
                for (int t = 0; t < 3; ++t) {
                    const int set = t / (16 / ROWS), c = t % (16 / ROWS) * ROWS + m;
                    reinterpret_cast<uint2*>(&s_dig[(k64 * SETS + set) * 64 + few_slot(k64, g, c)])[half] = d.digit[t];
                }
                if (run % 16 == 0) s_base[run / 16][m] = block_scale<ZERO>(top);
            }
        }
        lds_barrier();
        intx4 xf[NB][SETS][2];  // (columns of no row or digit hold anything: whole numbers that nobody reads)
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
                        else v = join_digits(p[0][r], p[1][r], p[2][r]);
                        sum[r] = u == 0 ? v * sc[j][i].get(r, u) : fmaf(v, sc[j][i].get(r, u), sum[r]);
                    }
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
                    if (SETS <= 1) v += s_red[buf][w][(out_m + 2 * ROWS) * 16 + out_row];
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

// ---- more rows -------------------------------------------------------------------------------------------------
// x as digits for the whole launch: digits [rows/16][Kpad/64][3][64 lanes][16 B], scales [rows/16][Kpad/128][16] fp32
struct Digits {
    uint8_t* d = nullptr;
    float* scale = nullptr;
};
// a thread per run of 8
template <bool ZERO>
__global__ __launch_bounds__(256) void digits_kernel(const float* __restrict__ x, int M, Linear4 l, Digits dg) {
    const int kb = l.Kpad / 128, run = blockIdx.x * 256 + threadIdx.x;
    const int64_t m = blockIdx.y;  // rows behind M: zeros
    if (run >= kb * 16) return;
    float v[8];
    load_run(x + (m < M ? m : M - 1) * l.K, run * 8, l.K, v);
    if (m >= M)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    const uint32_t top = block_top(v);
    const Run d = digits_of(v, top);
    const int step = run / 8, half = run / 4 % 2, g = run % 4;
    const int64_t mt = m / 16;
#pragma unroll
    for (int t = 0; t < 3; ++t)
        *reinterpret_cast<uint2*>(dg.d + (((mt * kb * 2 + step) * 3 + t) * 64 + g * 16 + m % 16) * 16 + half * 8) = d.digit[t];
    if (run % 16 == 0) dg.scale[(mt * kb + run / 16) * 16 + m % 16] = block_scale<ZERO>(top);
}

// A workgroup of 8 waves owns 256 columns (two tiles a wave), MT tiles of 16 rows and a slice of K, whose digits and scales pass
// through LDS block by block; slices go to `part` and are added by the caller's next launch.
template <int GROUP, bool ZERO, int MT>
__global__ __launch_bounds__(512, 2) void linear4_kernel(Linear4 l, Digits dg, int mt0, int M, int slice_blocks, float* __restrict__ out, int add) {
    constexpr int PER = 128 / GROUP, NT = 2, PIECES = MT * 384, NS = MT * 16;
    __shared__ uint4 s_dig[2][PIECES];
    __shared__ float s_scale[2][NS];
    const int lane = threadIdx.x & 63, col = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kb = l.Kpad / 128, tiles = (l.N + 15) / 16;
    const int b0 = blockIdx.y * slice_blocks, b1 = min(kb, b0 + slice_blocks);
    const int tile0 = (blockIdx.x * 8 + wave) * NT;
    float acc[NT][MT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[n][m][r] = 0.f;
    // block b of the MT row tiles, 6 KiB each, and their scales: three pieces of 16 bytes a thread or fewer
    uint4 stage0, stage1 = make_uint4(0, 0, 0, 0), stage2 = make_uint4(0, 0, 0, 0);
    float stage_s = 0.f;
    const int tid = threadIdx.x;
    const int j0 = min(tid, PIECES - 1), j1 = min(512 + tid, PIECES - 1), j2 = min(1024 + tid, PIECES - 1), js = min(tid, NS - 1);
    const uint8_t* x0 = dg.d + (int64_t)(mt0 + j0 / 384) * kb * 6144 + j0 % 384 * 16;
    const uint8_t* x1 = dg.d + (int64_t)(mt0 + j1 / 384) * kb * 6144 + j1 % 384 * 16;
    const uint8_t* x2 = dg.d + (int64_t)(mt0 + j2 / 384) * kb * 6144 + j2 % 384 * 16;
    const float* xs = dg.scale + (int64_t)(mt0 + js / 16) * kb * 16 + js % 16;
    auto load_x = [&](int b) {
        stage0 = *reinterpret_cast<const uint4*>(x0 + (int64_t)b * 6144);
        if (PIECES > 512) stage1 = *reinterpret_cast<const uint4*>(x1 + (int64_t)b * 6144);
        if (PIECES > 1024) stage2 = *reinterpret_cast<const uint4*>(x2 + (int64_t)b * 6144);
        stage_s = xs[(int64_t)b * 16];
    };
    auto store_x = [&](int buf) {
        s_dig[buf][tid] = stage0;
        if (PIECES > 512 && (PIECES >= 1024 || tid < PIECES - 512)) s_dig[buf][512 + tid] = stage1;
        if (PIECES > 1024 && (PIECES >= 1536 || tid < PIECES - 1024)) s_dig[buf][1024 + tid] = stage2;
        if (tid < NS) s_scale[buf][tid] = stage_s;
    };
    static_assert(PIECES >= 512 && PIECES <= 1536, "two to four row tiles");
    uint4 w[NT], wn[NT];
    uint32_t z[NT], zn[NT];
    Scales<GROUP> sc[NT], sn[NT];
    auto load_w = [&](int b) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int64_t tb = (int64_t)min(tile0 + n, tiles - 1) * kb + b;
            wn[n] = *reinterpret_cast<const uint4*>(l.w + (tb * 64 + lane) * 16);
            sn[n].load(l.scale, tb, g4);
            if (ZERO) zn[n] = load_zeros<GROUP>(l.zero, tb, col);
        }
    };
    load_w(b0);
    load_x(b0);
    store_x(0);
    int buf = 0;
    for (int b = b0; b < b1; ++b) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            w[n] = wn[n];
            if (ZERO) z[n] = zn[n];
            sc[n] = sn[n];
        }
        const int next = min(b + 1, b1 - 1);  // (the last block once more, not used)
        load_w(next);
        load_x(next);
        lds_barrier();
        intx4 a[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) unpack_block<GROUP, ZERO>(w[n], z[n], a[n]);
        intx4 xf[2][3][2];  // a row tile's operands are read while the one before it is multiplied
        float sx[2];
        auto read_x = [&](int m, intx4 (&f)[3][2], float& sxm) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < 3; ++t) f[t][h] = *reinterpret_cast<const intx4*>(&s_dig[buf][(m * 6 + h * 3 + t) * 64 + lane]);
            sxm = s_scale[buf][m * 16 + col];
        };
        read_x(0, xf[0], sx[0]);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m + 1 < MT) read_x(m + 1, xf[(m + 1) & 1], sx[(m + 1) & 1]);
            float sum[NT][4];
#pragma unroll
            for (int u = 0; u < PER; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    intx4(&f)[3][2] = xf[m & 1];
                    const intx4 p2 = group_product<GROUP>(a[n], f[0], u), p1 = group_product<GROUP>(a[n], f[1], u), p0 = group_product<GROUP>(a[n], f[2], u);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float v = join_digits(p2[r], p1[r], p0[r]);
                        sum[n][r] = u == 0 ? v * sc[n].get(r, u) : fmaf(v, sc[n].get(r, u), sum[n][r]);
                    }
                }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[n][m][r] = fmaf(sum[n][r], sx[m & 1], acc[n][m][r]);
                // one row tile at a time: left to itself the compiler keeps every tile's products for the end, and they do not fit the registers
                asm volatile("" : "+v"(acc[n][m][0]), "+v"(acc[n][m][1]), "+v"(acc[n][m][2]), "+v"(acc[n][m][3]));
            }
        }
        buf ^= 1;
        store_x(buf);  // read again only behind the next barrier; last read before this one
    }
    float* dst = out + (int64_t)blockIdx.y * M * l.N;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int64_t row = (int64_t)(mt0 + m) * 16 + col;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t c = (int64_t)(tile0 + n) * 16 + 4 * g4 + r;
                if (row < M && c < l.N) dst[row * l.N + c] = add ? dst[row * l.N + c] + acc[n][m][r] : acc[n][m][r];
            }
        }
}

// How a call of M rows runs: up to 16 by the few-row kernel; more by tiles of up to 64 rows, K sliced until the chip has a workgroup
// of 256 columns for every CU, each slice at least 4 blocks of 128.
struct Plan4 {
    int sets = 0, nb = 0, wgs = 0;  // few rows: operands, blocks per wave and chunk, workgroups per slice
    int row_tiles = 0, slices = 1, slice_blocks = 0;
    int64_t digit_bytes = 0, scale_bytes = 0, part_bytes = 0;
    int64_t bytes() const { return digit_bytes + scale_bytes + part_bytes; }
};
static Plan4 plan_linear4(const Linear4& l, int64_t M) {
    Plan4 p;
    const int64_t kb = l.Kpad / 128;
    if (M <= 16) {
        p.sets = M <= 4 ? 1 : M <= 8 ? 2 : 3;
        const int64_t most = p.sets == 3 || (p.sets == 2 && l.group == 32) ? 2 : p.sets == 2 || l.group < 128 ? 4 : 8;  // what LDS and registers hold
        const int64_t tiles = ((int64_t)l.N + 15) / 16;
        int64_t best = 0;
        for (int64_t s = 1; s <= 16; s *= 2) {
            if (s > 1 && kb / s < 4) break;
            // us, from single measurements: x into a CU at 45 B/ns and its conversion, for each workgroup a CU gets; the weights at a
            // CU's share of 6 TB/s; a second launch for slices and their traffic
            const int64_t blocks = (kb + s - 1) / s, room = kNumCU / s;
            const double rounds = (double)((tiles + room - 1) / room);
            const double turns = blocks > 8 * most && rounds > kFewTiles ? rounds / kFewTiles : 1.0;
            const double us = turns * (double)(blocks * 128 * M) * (4.0 / 45e3 + 4e-5) + rounds * (double)blocks * 1024 / 23.4e3 +
                              (s > 1 ? 5.0 + (double)s * (double)(M * l.N) * 8 / 4e6 : 0.0);
            static_assert(kNumCU % 16 == 0, "a slice's share of the CUs is a whole number");
            if (best == 0 || us * 1000 < (double)best) {
                best = (int64_t)(us * 1000);
                p.slices = (int)s;
            }
        }
        p.slice_blocks = (int)((kb + p.slices - 1) / p.slices);
        p.slices = (int)((kb + p.slice_blocks - 1) / p.slice_blocks);
        const int64_t chunks = (p.slice_blocks + 8 * most - 1) / (8 * most), need = (p.slice_blocks + 8 * chunks - 1) / (8 * chunks);
        p.nb = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 8;
        const int64_t room = std::max<int64_t>(1, kNumCU / p.slices);
        int64_t rounds = (tiles + room - 1) / room;
        if (p.slice_blocks > 8 * p.nb) rounds = std::min<int64_t>(rounds, kFewTiles);
        p.wgs = (int)((tiles + rounds - 1) / rounds);
    } else {
        const int64_t groups = ((int64_t)l.N + 255) / 256;
        p.row_tiles = (int)((M + 15) / 16);
        const int64_t passes = (M + 63) / 64, want = std::max<int64_t>(1, kNumCU / (groups * passes));
        const int64_t slices = std::min<int64_t>(want, std::max<int64_t>(1, kb / 4));
        p.slice_blocks = (int)((kb + slices - 1) / slices);
        p.slices = (int)((kb + p.slice_blocks - 1) / p.slice_blocks);
        p.digit_bytes = p.row_tiles * kb * 6144;
        p.scale_bytes = p.row_tiles * kb * 64;
    }
    if (p.slices > 1) p.part_bytes = p.slices * M * l.N * 4;
    return p;
}

template <int GROUP, bool ZERO>
static void launch_linear4(const Linear4& l, const float* x, int M, float* y, int accumulate, const Plan4& p, void* work, hipStream_t st) {
    float* part = (float*)((char*)work + p.digit_bytes + p.scale_bytes);
    float* out = p.slices > 1 ? part : y;
    const int add = p.slices > 1 ? 0 : accumulate;
    if (M <= 16) {
        const dim3 grid(p.wgs, p.slices);
        const bool one = p.wgs == (l.N + 15) / 16;
#define CHIRON_FEW(SETS_, NB_)                                                                                                                        \
    do {                                                                                                                                              \
        if (one) launch(linear4_few_kernel<GROUP, ZERO, SETS_, NB_, true>, grid, dim3(512), st, l, x, M, p.slice_blocks, out, add);              \
        else launch(linear4_few_kernel<GROUP, ZERO, SETS_, NB_, false>, grid, dim3(512), st, l, x, M, p.slice_blocks, out, add);                 \
    } while (0)
        if (p.sets == 1) {
            if (p.nb == 1) CHIRON_FEW(1, 1);
            else if (p.nb == 2) CHIRON_FEW(1, 2);
            else if (p.nb == 4 || GROUP < 128) CHIRON_FEW(1, 4);
            else if constexpr (GROUP == 128) CHIRON_FEW(1, 8);
        } else if (p.sets == 2) {
            if (p.nb == 1) CHIRON_FEW(2, 1);
            else if (p.nb == 2 || GROUP == 32) CHIRON_FEW(2, 2);
            else if constexpr (GROUP != 32) CHIRON_FEW(2, 4);
        } else {
            if (p.nb == 1) CHIRON_FEW(3, 1);
            else CHIRON_FEW(3, 2);
        }
#undef CHIRON_FEW
        return;
    }
    Digits dg;
    dg.d = (uint8_t*)work;
    dg.scale = (float*)(dg.d + p.digit_bytes);
    launch(digits_kernel<ZERO>, dim3((l.Kpad / 8 + 255) / 256, p.row_tiles * 16), dim3(256), st, x, M, l, dg);
    const dim3 grid((l.N + 255) / 256, p.slices);
    for (int mt = 0; mt < p.row_tiles;) {  // passes of nearly the same height, two tiles at least
        const int left = p.row_tiles - mt, passes = (left + 3) / 4, take = (left + passes - 1) / passes;
        if (take == 4) launch(linear4_kernel<GROUP, ZERO, 4>, grid, dim3(512), st, l, dg, mt, M, p.slice_blocks, out, add);
        else if (take == 3) launch(linear4_kernel<GROUP, ZERO, 3>, grid, dim3(512), st, l, dg, mt, M, p.slice_blocks, out, add);
        else launch(linear4_kernel<GROUP, ZERO, 2>, grid, dim3(512), st, l, dg, mt, M, p.slice_blocks, out, add);
        mt += take;
    }
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
    if (tiles * kb * 64 / 256 >= 0x7fffffff || kb * 128 > 0x7fffffff) return fail(CHIRON_ERR_SHAPE, "linear4: %d x %d is too large", N, K);
    chiron_linear4* l = new (std::nothrow) chiron_linear4();
    if (!l) return fail(CHIRON_ERR_OOM, "host allocation failed");
    Linear4& L = l->L;
    L.N = N; L.K = K; L.group = group; L.Kpad = (int)(kb * 128);
    const int64_t ns = tiles * 16 * (L.Kpad / group);
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
    if (p.slices > 1) return launch_reduce_partials((const float*)((char*)workspace + p.digit_bytes + p.scale_bytes), p.slices, (int64_t)M * L.N, y, accumulate, st);
    return CHIRON_OK;
}

}  // extern "C"
