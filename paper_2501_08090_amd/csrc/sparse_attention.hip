// Block-sparse attention of new tokens over the paged cache: score every page by its index record, take the best, attend over those.
// gfx950, wave64.
#include <algorithm>
#include <cmath>

#include "draft_ops.h"
#include "kv_layout.h"

namespace chiron {

typedef int intx4 __attribute__((ext_vector_type(4)));

// ---- scores -----------------------------------------------------------------------------------------------------
// score(p) = 2^e(p) * max_h sum_j (q8+[h][j] hi(p)[j] + q8-[h][j] lo(p)[j]): one product of length 2d per page and head, on the 8-bit
// matrix cores with whole-number accumulation.  A operand: 16 pages x 64 of the record's 2d codes; B: 16 columns, column c = query
// head c % G of the KV head.  Bounded by the records' bytes, (2d + 1) per page and head: 32 rows of some 28000 tokens, 8 KV heads of 128,
// 34 us with the selection (3.4 TB/s, 29 us where the last-level cache still holds them); one row of 8192 tokens 11 us, of which the
// scores take 3.7, the selection 2.5, the rest is the launch and a chain of loads.
struct SelectArgs {
    PoolDesc pool;
    IndexDesc index;
    const float* q;
    const int32_t *bt, *row_seq, *ctx_lens;
    float* scores;  // [rows][n_kv][max_blocks]
    int32_t *pages, *counts;
    int layer, max_blocks, top, n_first, n_last;
};

constexpr float kTop = 3.4028234663852886e38f;

// q8 of one (row, KV head) as B operand: column = head, 16 consecutive dims per lane group and step of 64; the positive ones first
template <int D, int G>
__device__ __forceinline__ void load_q8(const float* q, intx4 (&b)[D / 32]) {
    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const float* qp = q + (col % G) * D + g * 16;
    float x[D / 64][16], amax = 0.f;
#pragma unroll
    for (int s = 0; s < D / 64; ++s)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 v = *reinterpret_cast<const float4*>(qp + s * 64 + i);
            x[s][i] = finite_or(v.x, kTop);
            x[s][i + 1] = finite_or(v.y, kTop);
            x[s][i + 2] = finite_or(v.z, kTop);
            x[s][i + 3] = finite_or(v.w, kTop);
#pragma unroll
            for (int u = 0; u < 4; ++u) amax = fmaxf(amax, fabsf(x[s][i + u]));
        }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
    const float up = two_to(-power_of(amax));
#pragma unroll
    for (int s = 0; s < D / 64; ++s)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t pos = 0, neg = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int v = (int)rintf(x[s][w * 4 + i] * up);
                pos |= (uint32_t)max(v, 0) << (8 * i);
                neg |= (uint32_t)(min(v, 0) & 0xff) << (8 * i);
            }
            b[s][w] = (int)pos;
            b[s + D / 64][w] = (int)neg;
        }
}

// The scores of the 64 pages from p0 on, by one wave: the page that lane l's result belongs to is p0 + score_page(l).  All records
// (16 KiB at d = 128) are on their way before the first product.  block: lane l's is the pool's page of p0 + l, or of the last one.
__device__ __forceinline__ int score_page(int lane) { return (lane & 15) / 4 * 16 + (lane >> 4) * 4 + (lane & 3); }
template <int D>
__device__ __forceinline__ float score_64(const SelectArgs& a, int c, int block, const intx4 (&b)[D / 32]) {
    constexpr int KS = D / 32;  // steps of 64 codes: the first half meets the bounds from above, the second those from below
    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const bool bad = block < 0 || block >= a.pool.num_blocks;
    block = bad ? 0 : block;
    intx4 rec[4][KS];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int8_t* p = index_codes(a.index, a.layer, __shfl(block, 16 * t + col), c) + g * 16;  // A operand: row = lane % 16
#pragma unroll
        for (int s = 0; s < KS; ++s) rec[t][s] = *reinterpret_cast<const intx4*>(p + s * 64);
    }
    const int e = bad ? -1000 : *index_exp(a.index, a.layer, block, c);
    int mine = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        intx4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(rec[t][s], b[s], acc, 0, 0, 0);
        // accumulator: column = lane % 16, page 16t + 4g + r in register r; the maximum over the columns, in all 16 lanes
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            int m = acc[r];
            m = max(m, row_move<kRor8>(m));
            m = max(m, row_move<kRor4>(m));
            m = max(m, row_move<kRor2>(m));
            m = max(m, row_move<kRor1>(m));
            mine = col == 4 * t + r ? m : mine;
        }
    }
    const int em = __shfl(e, score_page(lane));
    return em == -1000 ? -kTop : finite_or((float)mine * two_to(em), kTop);
}

// Workgroup b works for list list_at(b): the lists of one row, one behind the other, run on one XCD (workgroups go to the eight in
// turn), whose L2 then serves the row's exponents, eight heads to a line, and page ids to all of them.
__device__ __forceinline__ int list_at(int b, int lists) {
    const int xcd = b & 7, each = lists >> 3, more = lists & 7;
    return xcd * each + min(xcd, more) + (b >> 3);
}
// what both forms of the selection begin with
struct ListOf {
    int n, c;
    const int32_t* btrow;
    const float* q;
};
template <int D, int G>
__device__ __forceinline__ ListOf list_of(const SelectArgs& a, int list) {
    ListOf l;
    const int row = list / a.pool.n_kv, ctx = a.ctx_lens[row], seq = a.row_seq ? a.row_seq[row] : row;
    l.c = list - row * a.pool.n_kv;
    l.n = ctx <= 0 ? 0 : (int)min(((int64_t)ctx + kBlockSize - 1) / kBlockSize, (int64_t)a.max_blocks);
    l.btrow = a.bt + (size_t)seq * a.max_blocks;
    l.q = a.q + (size_t)list * (G * D);
    return l;
}

// ---- the `top` best pages of a list, ascending -------------------------------------------------------------------
// By a workgroup.  Scores are order-preserving 32-bit keys.  Of the pages that are not forced, the key of the last one taken is found
// 8 bits at a time, from the first bit in which the list's keys differ on, with histograms in LDS; it ends early where a bin is taken
// whole.  Then every wave counts and writes what its run of pages holds.
__device__ __forceinline__ uint32_t score_key(float f) {
    const uint32_t u = __float_as_uint(f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
constexpr int kSelectThreads = 512, kSelectWaves = kSelectThreads / 64;
struct SelectShared {
    uint32_t hist[256];
    uint32_t lo[kSelectWaves], hi[kSelectWaves];
    uint32_t bin, before, inside;
    int gt[kSelectWaves], eq[kSelectWaves];
};
template <typename Key>
__device__ __forceinline__ void select_top(const SelectArgs& a, int n, const Key& key_of, SelectShared& sh, int32_t* out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int f0 = a.n_first, f1 = n - a.n_last;  // the pages f0 .. f1-1 compete
    uint32_t left = a.top - a.n_first - a.n_last;
    uint32_t from = 0xffffffffu, equal = 0xffffffffu;  // taken: keys >= from, and the first `left` at `equal` (no score has that key)
    if (left > 0) {
        uint32_t lo = 0xffffffffu, hi = 0;
        for (int p = f0 + threadIdx.x; p < f1; p += kSelectThreads) {
            const uint32_t k = key_of(p);
            lo = min(lo, k);
            hi = max(hi, k);
        }
#pragma unroll
        for (int o = 32; o >= 16; o >>= 1) {
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
        }
        lo = min(lo, (uint32_t)row_move<kRor8>((int)lo)), hi = max(hi, (uint32_t)row_move<kRor8>((int)hi));
        lo = min(lo, (uint32_t)row_move<kRor4>((int)lo)), hi = max(hi, (uint32_t)row_move<kRor4>((int)hi));
        lo = min(lo, (uint32_t)row_move<kRor2>((int)lo)), hi = max(hi, (uint32_t)row_move<kRor2>((int)hi));
        lo = min(lo, (uint32_t)row_move<kRor1>((int)lo)), hi = max(hi, (uint32_t)row_move<kRor1>((int)hi));
        if (lane == 0) {
            sh.lo[wave] = lo;
            sh.hi[wave] = hi;
        }
        if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSelectWaves; ++w) {
            lo = min(lo, sh.lo[w]);
            hi = max(hi, sh.hi[w]);
        }
        int bits = lo == hi ? 0 : 32 - __clz(lo ^ hi);  // the keys agree above them
        uint32_t prefix = hi;
        if (bits == 0) equal = hi, from = hi + 1;
        while (bits > 0) {
            const int shift = max(0, bits - 8);
            const uint32_t mask = (1u << (bits - shift)) - 1;
            for (int p = f0 + threadIdx.x; p < f1; p += kSelectThreads) {
                const uint32_t k = key_of(p);
                if (bits == 32 || k >> bits == prefix >> bits) atomicAdd(&sh.hist[k >> shift & mask], 1u);
            }
            __syncthreads();
            if (wave == 0) {
                // lane l holds the bins 255-4l .. 252-4l, from the top; the bin in which the running count reaches `left`
                uint32_t h[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[i] = sh.hist[255 - 4 * lane - i];
                    sum += h[i];
                }
                uint32_t before = (uint32_t)wave_scan((int)sum) - sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < left && before + h[i] >= left) {
                        sh.bin = 255 - 4 * lane - i;
                        sh.before = before;
                        sh.inside = h[i];
                    }
                    before += h[i];
                }
            }
            __syncthreads();
            const uint32_t inside = sh.inside;
            prefix = (bits == 32 ? 0 : prefix >> bits << bits) | sh.bin << shift;
            left -= sh.before;
            if (inside == left) {
                from = prefix;
                left = 0;
                break;
            }
            bits = shift;
            if (bits == 0) {
                equal = prefix;
                from = prefix + 1;
                break;
            }
            if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
            __syncthreads();
        }
    }
    // wave w has the pages [w0, w1)
    auto test = [&](int p, int w1, bool& gt, bool& eq) {
        const bool forced = p < f0 || p >= f1;
        const uint32_t k = p < w1 && !forced ? key_of(p) : 0;
        gt = p < w1 && (forced || k >= from);
        eq = p < w1 && !forced && k == equal;
    };
    const int run = (n + kSelectThreads - 1) / kSelectThreads * 64, w0 = min(n, wave * run), w1 = min(n, w0 + run);
    int n_gt = 0, n_eq = 0;
    for (int p = w0 + lane; p - lane < w1; p += 64) {
        bool gt, eq;
        test(p, w1, gt, eq);
        n_gt += __popcll(__ballot(gt));
        n_eq += __popcll(__ballot(eq));
    }
    if (lane == 0) {
        sh.gt[wave] = n_gt;
        sh.eq[wave] = n_eq;
    }
    __syncthreads();
    int gt0 = 0, eq0 = 0;
    for (int w = 0; w < wave; ++w) {
        gt0 += sh.gt[w];
        eq0 += sh.eq[w];
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    for (int p = w0 + lane; p - lane < w1; p += 64) {
        bool gt, eq;
        test(p, w1, gt, eq);
        const uint64_t bg = __ballot(gt), be = __ballot(eq);
        const int eqs = eq0 + __popcll(be & below);  // pages at `equal` before this one
        if (gt || (eq && eqs < (int)left)) out[gt0 + __popcll(bg & below) + min(eqs, (int)left)] = p;
        gt0 += __popcll(bg);
        eq0 += __popcll(be);
    }
}
// lists that take every page, and the counts
__device__ __forceinline__ bool select_all(const SelectArgs& a, int list, int n, int32_t* out) {
    if (a.counts && list % a.pool.n_kv == 0 && threadIdx.x == 0) a.counts[list / a.pool.n_kv] = min(n, a.top);
    if (n > a.top) return false;
    for (int i = threadIdx.x; i < a.top; i += kSelectThreads) out[i] = i < n ? i : -1;
    return true;
}

// One launch, a workgroup per (row, KV head) that scores its pages into LDS and selects: as long as one CU can take in a list's records
// in about the time of the second launch, or there are lists for half the CUs.  (Attention included: one row over 4096 tokens of 2 KV
// heads of 64 14.1 us, in two launches 15.5; over 32768 of 8 of 128 35, in two 24.9.)
constexpr int kSelectPages = 15360;  // keys that fit 64 KiB of LDS beside the rest
template <int D, int G>
__global__ __launch_bounds__(kSelectThreads, 2) void select_pages_kernel(SelectArgs a) {
    __shared__ SelectShared sh;
    extern __shared__ uint32_t s_keys[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, list = list_at(blockIdx.x, gridDim.x);
    const ListOf l = list_of<D, G>(a, list);
    int32_t* out = a.pages + (size_t)list * a.top;
    if (select_all(a, list, l.n, out)) return;
    intx4 b[D / 32];
    int block = l.btrow[min(wave * 64 + lane, l.n - 1)];  // one step ahead
    load_q8<D, G>(l.q, b);
    for (int p0 = wave * 64; p0 < l.n; p0 += kSelectThreads) {
        const int next = l.btrow[min(p0 + kSelectThreads + lane, l.n - 1)];
        const float f = score_64<D>(a, l.c, block, b);
        block = next;
        s_keys[p0 + score_page(lane)] = score_key(f);  // (the places up to the next multiple of 64 are there)
    }
    __syncthreads();
    select_top(a, l.n, [&](int p) { return s_keys[p]; }, sh, out);
}

// Two launches: few and long lists are scored by many workgroups, through memory
template <int D, int G>
__global__ __launch_bounds__(256) void page_scores_kernel(SelectArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, list = list_at(blockIdx.x, gridDim.x);
    const ListOf l = list_of<D, G>(a, list);
    if (l.n <= a.top) return;  // every page is taken: nobody reads the scores
    intx4 b[D / 32];
    const int first = (blockIdx.y * 4 + wave) * 64, step = gridDim.y * 256;
    int block = l.btrow[min(first + lane, l.n - 1)];  // one step ahead
    load_q8<D, G>(l.q, b);
    float* out = a.scores + (size_t)list * a.max_blocks;
    for (int p0 = first; p0 < l.n; p0 += step) {
        const int next = l.btrow[min(p0 + step + lane, l.n - 1)];
        const float f = score_64<D>(a, l.c, block, b);
        block = next;
        const int p = p0 + score_page(lane);
        if (p < l.n) out[p] = f;
    }
}
__global__ __launch_bounds__(kSelectThreads) void select_scored_kernel(SelectArgs a) {
    __shared__ SelectShared sh;
    const int list = blockIdx.x, ctx = a.ctx_lens[list / a.pool.n_kv];
    const int n = ctx <= 0 ? 0 : (int)min(((int64_t)ctx + kBlockSize - 1) / kBlockSize, (int64_t)a.max_blocks);
    int32_t* out = a.pages + (size_t)list * a.top;
    if (select_all(a, list, n, out)) return;
    const float* scores = a.scores + (size_t)list * a.max_blocks;
    select_top(a, n, [&](int p) { return score_key(scores[p]); }, sh, out);
}

// ---- attention over listed pages -----------------------------------------------------------------------------------
// A wave streams the pages of its part of a list (K and V tiles straight into matrix-core operands, as the pool's layout gives them)
// with a running maximum and sum.  q and P enter as three bf16 terms (24 bits): with few heads per KV head the terms of one head
// take different operand columns of one instruction, column = group * G + head, and the sums over the groups are rotations within
// 16 lanes.  The waves of a workgroup take parts of one list and merge in LDS; a list may be split over `splits` workgroups, whose
// partial results a second kernel joins (selection included, one row over 8192 tokens, 64 pages of 8 lists: 21.1 us, unsplit 23.1; over
// 32768: 24.9 and 30.3).  Bound by the pages' bytes: 32 rows x 8 lists of 128 pages of 8 KiB 49 us (5.4 TB/s); one row 9 us, a chain of
// loads: the list, the block table, keys and values.
constexpr int kSparseWaves = 8;
template <int D, int G>
__global__ __launch_bounds__(kSparseWaves * 64, 2) void sparse_attn_kernel(PoolDesc pool, int layer, const float* __restrict__ q,
                                                                          const int32_t* __restrict__ bt, int max_blocks,
                                                                          const int32_t* __restrict__ row_seq,
                                                                          const int32_t* __restrict__ ctx_lens,
                                                                          const int32_t* __restrict__ pages,
                                                                          const int32_t* __restrict__ counts, int top, int splits,
                                                                          float scale_log2e, float* __restrict__ out,
                                                                          float* __restrict__ part_o, float* __restrict__ part_ml) {
    constexpr int KSTEPS = D / 32, NPG = 2;
    constexpr int GROUPS = 16 / G, TPI = GROUPS < 3 ? GROUPS : 3;  // terms that fit one instruction
    constexpr int NI = (3 + TPI - 1) / TPI;                         // instructions for the three terms
    __shared__ float s_o[kSparseWaves][G][D];
    __shared__ float s_ml[kSparseWaves][G][2];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_kv = pool.n_kv;
    const int split = blockIdx.x % splits, rc = blockIdx.x / splits, row = rc / n_kv, c = rc % n_kv;
    const int head = lane & 15, lg = lane >> 4, h = head % G, grp = head / G;
    const int len = (int)min((int64_t)ctx_lens[row], (int64_t)max_blocks * kBlockSize);
    const int listed = min(counts ? max(counts[row], 0) : top, top);
    const int parts = splits * kSparseWaves, mine = split * kSparseWaves + wave;
    const int i0 = (int)((int64_t)listed * mine / parts), i1 = (int)((int64_t)listed * (mine + 1) / parts);
    const int32_t* list = pages + (size_t)rc * top;
    const int seq = row_seq ? row_seq[row] : row;
    const int32_t* btrow = bt + (size_t)seq * max_blocks;
    const uint16_t* lbase = pool.base + (size_t)layer * (size_t)pool.layer_stride;
    constexpr size_t tile_elems = (size_t)16 * D;

    floatx4 o[D / 16];
#pragma unroll
    for (int t = 0; t < D / 16; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    if (i0 < i1) {
        // the terms of a value that this lane's column takes, for instruction j
        auto term = [&](float v, int j) {
            const float hi = bf16_lo(pack_bf16_rne(v, 0.f));
            const float r1 = v - hi, mid = bf16_lo(pack_bf16_rne(r1, 0.f)), lo = r1 - mid;
            const int t = j * TPI + grp;
            return grp >= TPI ? 0.f : t == 0 ? hi : t == 1 ? mid : t == 2 ? lo : 0.f;
        };
        uint4 qt[NI][KSTEPS];
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            const float* qp = q + ((size_t)rc * G + h) * D + s * 32 + lg * 8;
            const float4 a = *reinterpret_cast<const float4*>(qp), b = *reinterpret_cast<const float4*>(qp + 4);
            const float x[8] = {a.x * scale_log2e, a.y * scale_log2e, a.z * scale_log2e, a.w * scale_log2e,
                                b.x * scale_log2e, b.y * scale_log2e, b.z * scale_log2e, b.w * scale_log2e};
#pragma unroll
            for (int j = 0; j < NI; ++j)
                qt[j][s] = make_uint4(pack_bf16_rne(term(x[0], j), term(x[1], j)), pack_bf16_rne(term(x[2], j), term(x[3], j)),
                                      pack_bf16_rne(term(x[4], j), term(x[5], j)), pack_bf16_rne(term(x[6], j), term(x[7], j)));
        }
        // lane l holds entry base + l of the list: the page and where it is in the pool
        int base = i0, v_page, v_block;
        auto fetch = [&] {
            const int i = base + lane;
            int pg = i < i1 ? list[i] : -1;
            if (pg < 0 || pg >= max_blocks || (int64_t)pg * kBlockSize >= len) pg = -1;
            int blk = pg >= 0 ? btrow[pg] : -1;
            if (blk < 0 || blk >= pool.num_blocks) pg = -1;
            v_page = pg;
            v_block = pg >= 0 ? blk : 0;  // an entry that counts for nothing reads page 0 of the pool and masks all of it
        };
        fetch();
        uint4 kc[NPG][KSTEPS], vc[NPG][KSTEPS], kn[NPG][KSTEPS], vn[NPG][KSTEPS];
        int pc[NPG], pn[NPG];
        auto load_group = [&](int i, uint4 (&kk)[NPG][KSTEPS], uint4 (&vv)[NPG][KSTEPS], int (&pg)[NPG]) {
#pragma unroll
            for (int u = 0; u < NPG; ++u) {
                const int at = i + u - base;  // uniform
                const bool on = i + u < i1;
                pg[u] = on ? __builtin_amdgcn_readlane(v_page, at & 63) : -1;
                const int blk = on ? __builtin_amdgcn_readlane(v_block, at & 63) : 0;
                const uint16_t* tile = lbase + ((size_t)blk * n_kv + c) * (2 * tile_elems);
#pragma unroll
                for (int s = 0; s < KSTEPS; ++s) {
                    kk[u][s] = load_stream_16(tile + (size_t)(s * 64 + lane) * 8);
                    vv[u][s] = load_stream_16(tile + tile_elems + (size_t)(s * 64 + lane) * 8);
                }
            }
        };
        auto compute = [&] {
            floatx4 s[NPG];
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < NPG; ++u) {
                s[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
                    for (int j = 0; j < NI; ++j)
                        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<bf16x8*>(&kc[u][k]), *reinterpret_cast<bf16x8*>(&qt[j][k]), s[u], 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) {  // the sum over the column groups, in every column of a head
                    if (G <= 8) s[u][r] += row_move<kRor8>(s[u][r]);
                    if (G <= 4) s[u][r] += row_move<kRor4>(s[u][r]);
                    if (G <= 2) s[u][r] += row_move<kRor2>(s[u][r]);
                    if (G <= 1) s[u][r] += row_move<kRor1>(s[u][r]);
                }
                const int left = pc[u] < 0 ? 0 : len - pc[u] * kBlockSize;  // tokens of the page that count (uniform)
                if (left < kBlockSize) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[u][r] = lg * 4 + r < left ? s[u][r] : -INFINITY;
                    // what other slots hold may be anything, NaN included: clear their V so that 0 * V stays 0
                    const int valid = left - lg * 4;
                    const uint32_t m01 = (valid > 0 ? 0x0000ffffu : 0u) | (valid > 1 ? 0xffff0000u : 0u);
                    const uint32_t m23 = (valid > 2 ? 0x0000ffffu : 0u) | (valid > 3 ? 0xffff0000u : 0u);
#pragma unroll
                    for (int k = 0; k < KSTEPS; ++k) {
                        vc[u][k].x &= m01; vc[u][k].y &= m23; vc[u][k].z &= m01; vc[u][k].w &= m23;
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[u][r]);
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_run, mx), m_use = fmaxf(m_new, -1e30f);  // nothing seen yet: finite exponents, weights 0
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) o[t] *= alpha;
#pragma unroll
            for (int u = 0; u < NPG; ++u) {
                float pr[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    pr[r] = __builtin_amdgcn_exp2f(s[u][r] - m_use);
                    l_run += pr[r];
                }
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    uint2 pt = make_uint2(pack_bf16_rne(term(pr[0], j), term(pr[1], j)), pack_bf16_rne(term(pr[2], j), term(pr[3], j)));
                    const short4v b = *reinterpret_cast<short4v*>(&pt);
#pragma unroll
                    for (int k = 0; k < KSTEPS; ++k) {
                        uint2 v0 = make_uint2(vc[u][k].x, vc[u][k].y), v1 = make_uint2(vc[u][k].z, vc[u][k].w);
                        o[2 * k] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(*reinterpret_cast<short4v*>(&v0), b, o[2 * k], 0, 0, 0);
                        o[2 * k + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(*reinterpret_cast<short4v*>(&v1), b, o[2 * k + 1], 0, 0, 0);
                    }
                }
            }
        };
        load_group(i0, kc, vc, pc);
        for (int i = i0; i < i1; i += NPG) {
            if (i + NPG < i1) {
                if (i + NPG - base >= 64) {  // uniform; 64 is a multiple of NPG
                    base = i + NPG;
                    fetch();
                }
                load_group(i + NPG, kn, vn, pn);
            }
            __builtin_amdgcn_sched_barrier(0);
            compute();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < NPG; ++u) {
                pc[u] = pn[u];
#pragma unroll
                for (int k = 0; k < KSTEPS; ++k) {
                    kc[u][k] = kn[u][k];
                    vc[u][k] = vn[u][k];
                }
            }
        }
        l_run += __shfl_xor(l_run, 16);
        l_run += __shfl_xor(l_run, 32);
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (G <= 8) o[t][r] += row_move<kRor8>(o[t][r]);
                if (G <= 4) o[t][r] += row_move<kRor4>(o[t][r]);
                if (G <= 2) o[t][r] += row_move<kRor2>(o[t][r]);
                if (G <= 1) o[t][r] += row_move<kRor1>(o[t][r]);
            }
    }
    if (head < G) {
        if (lg == 0) {
            s_ml[wave][head][0] = m_run;
            s_ml[wave][head][1] = l_run;
        }
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
            *reinterpret_cast<float4*>(&s_o[wave][head][t * 16 + lg * 4]) = make_float4(o[t][0], o[t][1], o[t][2], o[t][3]);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < G * D; e += kSparseWaves * 64) {
        const int a = e / D, j = e % D;
        float M = -1e30f;
#pragma unroll
        for (int w = 0; w < kSparseWaves; ++w) M = fmaxf(M, s_ml[w][a][0]);
        float num = 0.f, den = 0.f;
#pragma unroll
        for (int w = 0; w < kSparseWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_ml[w][a][0] - M);
            num += f * s_o[w][a][j];
            den += f * s_ml[w][a][1];
        }
        if (splits == 1) out[((size_t)rc * G + a) * D + j] = den > 0.f ? num / den : 0.f;
        else {
            const size_t slot = ((size_t)rc * splits + split) * G + a;
            part_o[slot * D + j] = num;
            if (j == 0) {
                part_ml[slot * 2] = M;
                part_ml[slot * 2 + 1] = den;
            }
        }
    }
}

// joins the splits of a list: a thread per (row, query head, dim)
template <int D>
__global__ __launch_bounds__(256) void sparse_merge_kernel(const float* __restrict__ part_o, const float* __restrict__ part_ml, int G, int splits,
                                                           int64_t n, float* __restrict__ out) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= n) return;
    const int64_t rh = j / D;  // (row, KV head, head of the group)
    const int e = (int)(j % D), a = (int)(rh % G);
    const int64_t slot0 = rh / G * splits * G + a;
    float M = -1e30f, num = 0.f, den = 0.f;
    constexpr int kAtOnce = 8;  // splits whose loads are on their way together
    for (int s0 = 0; s0 < splits; s0 += kAtOnce) {
        float2 ml[kAtOnce];
        float o[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int64_t slot = slot0 + (int64_t)min(s0 + i, splits - 1) * G;
            ml[i] = *reinterpret_cast<const float2*>(part_ml + slot * 2);
            o[i] = part_o[slot * D + e];
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, ml[i].x);
        const float keep = __builtin_amdgcn_exp2f(M - top);
        M = top;
        num *= keep;
        den *= keep;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const float f = s0 + i < splits ? __builtin_amdgcn_exp2f(ml[i].x - M) : 0.f;
            num += f * o[i];
            den += f * ml[i].y;
        }
    }
    out[j] = den > 0.f ? num / den : 0.f;
}

static int32_t check_sparse(const chiron_model* m, const chiron_kvpool* p, int32_t layer, int32_t rows, int32_t top) {
    if (!m || !p) return fail(CHIRON_ERR_INVALID_ARG, "model or pool is null");
    if (rows < 0) return fail(CHIRON_ERR_INVALID_ARG, "rows is negative");
    if (rows > m->cfg.max_batch) return fail(CHIRON_ERR_BATCH_TOO_LARGE, "rows %d exceed max_batch %d", rows, m->cfg.max_batch);
    if (p->d.n_kv != m->cfg.n_kv_heads || p->d.d != m->cfg.head_dim || p->d.n_layers != m->cfg.n_layers)
        return fail(CHIRON_ERR_INVALID_ARG, "pool was created for a different model shape");
    if (layer < 0 || layer >= p->d.n_layers) return fail(CHIRON_ERR_INVALID_ARG, "layer %d out of range", layer);
    if (top < 1) return fail(CHIRON_ERR_INVALID_ARG, "top %d: at least one page is taken", top);
    return CHIRON_OK;
}

#define CHIRON_BY_HEADS(CALL, D_)                                                                                       \
    switch (G) {                                                                                                        \
        case 1: CALL(D_, 1); break;                                                                                     \
        case 2: CALL(D_, 2); break;                                                                                     \
        case 4: CALL(D_, 4); break;                                                                                     \
        case 8: CALL(D_, 8); break;                                                                                     \
        case 16: CALL(D_, 16); break;                                                                                   \
        default: return fail(CHIRON_ERR_SHAPE, "query heads per KV head must be 1, 2, 4, 8 or 16 (got %d)", G);         \
    }

}  // namespace chiron

using namespace chiron;

extern "C" {

int32_t chiron_op_select_pages(chiron_model* m, const chiron_kvpool* p, const chiron_kvindex* x, int32_t layer, const float* q,
                               const int32_t* block_table, const int32_t* row_seq, const int32_t* ctx_lens, int32_t rows, int32_t top,
                               int32_t n_first, int32_t n_last, int32_t* pages, int32_t* counts, void* stream) {
    int32_t rc = check_sparse(m, p, layer, rows, top);
    if (rc) return rc;
    if (!x) return fail(CHIRON_ERR_INVALID_ARG, "page index is null");
    if (!index_fits(x->d, p->d)) return fail(CHIRON_ERR_INVALID_ARG, "the page index was created for another pool shape");
    if (n_first < 0 || n_last < 0 || (int64_t)n_first + n_last > top)
        return fail(CHIRON_ERR_INVALID_ARG, "select: n_first %d and n_last %d must be >= 0 and at most top %d together", n_first, n_last, top);
    if (rows == 0) return CHIRON_OK;
    if (!q || !block_table || !ctx_lens || !pages) return fail(CHIRON_ERR_INVALID_ARG, "select: a pointer is null");
    if ((uintptr_t)q & 15) return fail(CHIRON_ERR_INVALID_ARG, "select: q must be 16-byte aligned");
    const int n_kv = p->d.n_kv, G = m->cfg.n_q_heads / n_kv, mb = m->cfg.max_blocks_per_seq;
    const int64_t lists = (int64_t)rows * n_kv;
    if (lists > 0x7fffffff) return fail(CHIRON_ERR_BATCH_TOO_LARGE, "select: %lld lists are too many", (long long)lists);
    SelectArgs a;
    a.pool = p->d; a.index = x->d; a.q = q; a.bt = block_table; a.row_seq = row_seq; a.ctx_lens = ctx_lens; a.scores = m->aws.part_o;
    a.pages = pages; a.counts = counts; a.layer = layer; a.max_blocks = mb; a.top = top; a.n_first = n_first; a.n_last = n_last;
    hipStream_t st = (hipStream_t)stream;
    const int d = p->d.d;
    // us of a CU for a whole list's records at 45 B/ns, against some 5 us for the second launch.  The host knows the table's width, not what
    // the rows see of it, and short lists cost less in the wrong form than long ones: us in one launch / two, 8 KV heads of 128, tables of
    // 8192 columns: one row of 100 pages 7.0 / 8.8, 510 10.7 / 10.8, 2000 23.6 / 13.8; 4 rows 7.3 / 11.4, 10.7 / 12.8, 23.8 / 16.7; 15 rows 7.3 /
    // 11.5, 10.9 / 13.6, 26.4 / 24.9.
    const bool one = mb <= kSelectPages && (lists * 2 >= kNumCU || (double)mb * 2 * d / 45e3 <= 5.0);
    if (one) {
        const size_t lds = ((size_t)mb + 63) / 64 * 64 * 4;
#define CHIRON_SELECT(D_, G_) launch_lds(select_pages_kernel<D_, G_>, dim3((unsigned)lists), dim3(kSelectThreads), lds, st, a)
        if (d == 128) CHIRON_BY_HEADS(CHIRON_SELECT, 128)
        else CHIRON_BY_HEADS(CHIRON_SELECT, 64)
#undef CHIRON_SELECT
    } else {
        // The scores lie in the attention workspace: as many rows at once as it holds, one range behind the other on the stream.
        const int64_t at_once = (int64_t)m->aws.cap_items * m->cfg.n_q_heads * d / ((int64_t)n_kv * mb);
        if (at_once < 1) return fail(CHIRON_ERR_SHAPE, "select: scores of %d heads x %d pages exceed the model's workspace", n_kv, mb);
        for (int64_t r0 = 0; r0 < rows; r0 += at_once) {
            const int64_t n = std::min<int64_t>(at_once, rows - r0), part = n * n_kv;
            a.q = q + r0 * m->cfg.n_q_heads * d;
            a.ctx_lens = ctx_lens + r0;
            a.row_seq = row_seq ? row_seq + r0 : nullptr;
            a.bt = row_seq ? block_table : block_table + r0 * mb;
            a.pages = pages + r0 * n_kv * top;
            a.counts = counts ? counts + r0 : nullptr;
            const int chunks = (int)std::min<int64_t>((mb + 255) / 256, std::max<int64_t>(1, 4 * kNumCU / part));
            const dim3 grid((unsigned)part, chunks);
            if (mb > top) {
#define CHIRON_SCORES(D_, G_) launch(page_scores_kernel<D_, G_>, grid, dim3(256), st, a)
                if (d == 128) CHIRON_BY_HEADS(CHIRON_SCORES, 128)
                else CHIRON_BY_HEADS(CHIRON_SCORES, 64)
#undef CHIRON_SCORES
            }
            launch(select_scored_kernel, dim3((unsigned)part), dim3(kSelectThreads), st, a);
        }
    }
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

int32_t chiron_op_sparse_attention(chiron_model* m, const chiron_kvpool* p, int32_t layer, const float* q, const int32_t* block_table,
                                   const int32_t* row_seq, const int32_t* ctx_lens, int32_t rows, const int32_t* pages,
                                   const int32_t* counts, int32_t top, float* out, void* stream) {
    int32_t rc = check_sparse(m, p, layer, rows, top);
    if (rc) return rc;
    if (rows == 0) return CHIRON_OK;
    if (!q || !block_table || !ctx_lens || !pages || !out) return fail(CHIRON_ERR_INVALID_ARG, "sparse attention: a pointer is null");
    if (((uintptr_t)q | (uintptr_t)out) & 15) return fail(CHIRON_ERR_INVALID_ARG, "sparse attention: q and out must be 16-byte aligned");
    const int n_kv = p->d.n_kv, n_q = m->cfg.n_q_heads, G = n_q / n_kv, d = p->d.d, mb = m->cfg.max_blocks_per_seq;
    const int64_t lists = (int64_t)rows * n_kv;
    // a workgroup per list and split: enough of them for one round of the chip, each wave at least two pages
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(top / (2 * kSparseWaves), m->aws.cap_items / rows));
    const int splits = (int)std::min<int64_t>(most, std::max<int64_t>(1, kNumCU / lists));
    if (lists * splits > 0x7fffffff || lists * G * d / 256 > 0x7ffffff0) return fail(CHIRON_ERR_BATCH_TOO_LARGE, "sparse attention: %lld lists are too many", (long long)lists);
    const float scale = (float)(1.4426950408889634 / std::sqrt((double)d));
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)(lists * splits));
#define CHIRON_SPARSE(D_, G_)                                                                                                           \
    launch(sparse_attn_kernel<D_, G_>, grid, dim3(kSparseWaves * 64), st, p->d, layer, q, block_table, mb, row_seq, ctx_lens, pages, counts, top, \
           splits, scale, out, m->aws.part_o, m->aws.part_ml)
    if (d == 128) CHIRON_BY_HEADS(CHIRON_SPARSE, 128)
    else CHIRON_BY_HEADS(CHIRON_SPARSE, 64)
#undef CHIRON_SPARSE
    if (splits > 1) {
        const int64_t n = (int64_t)rows * n_q * d;
        const dim3 g((unsigned)((n + 255) / 256));
        if (d == 128) launch(sparse_merge_kernel<128>, g, dim3(256), st, m->aws.part_o, m->aws.part_ml, G, splits, n, out);
        else launch(sparse_merge_kernel<64>, g, dim3(256), st, m->aws.part_o, m->aws.part_ml, G, splits, n, out);
    }
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

}  // extern "C"
