// Attention of new rows over the paged cache, bf16 or 8 bits: causal, within a window and over first tokens that stay visible.  gfx950,
// wave64.
//
// Both kernels hold the scores transposed, tokens as rows and (row, query head) pairs of one KV head as columns, 16 x 16 at a time
// (v_mfma_f32_16x16x32_bf16): a score tile's registers are then the operand that the product with V wants, the running maximum and sum
// of a softmax belong to a lane's column, and a row's queries that share a KV head share one pass over its pages.  An 8-bit code is
// widened to bf16 in registers, exactly; its power of two goes to the score (keys) or the weight (values).
//
// fp32 queries enter as three bf16 terms, and so do the weights: 24 bits, which keeps fp32's accuracy.  bf16 queries are one term,
// their weights two where requests bring few rows (memory is what those wait for: the same time) and one, rounded, in prompts (whose errors are
// then up to 1.4 times those of out's own rounding; a second term would be a second product with V).
#include <algorithm>
#include <array>
#include <cmath>
#include <type_traits>

#include "cache8.h"
#include "kv_layout.h"

namespace chiron {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct RowAttnArgs {
    const uint8_t* tiles;  // the layer's: [num_blocks][n_kv][K tile, V tile]
    const int8_t* exps;    // 8-bit pools: [num_blocks][n_kv][K, V]
    const void* q;
    void* out;
    int64_t q_stride;  // elements
    const int32_t *bt, *row_starts, *seq_lens;
    int64_t window;
    int num_blocks, n_kv, G, max_blocks, batch, rows, max_new, n_sinks;
    float scale_log2e;
    int few_max;      // requests of at most so many rows are row_few_kernel's (0: none), the others row_many_kernel's
    int tg, pcols;    // tokens that share a pass of row_few_kernel, and the columns of a partial result
    int passes_max;   // no more passes than this
    int tt, splits;   // tokens of a tile of row_many_kernel, parts of its pages
    int32_t* head;    // [0]: passes; then a record of four for each pass: first row, tokens, first partial result, partial results
    float *part_o, *part_ml;
    float *many_o, *many_ml;
};

// ---- what a row sees --------------------------------------------------------------------------------------------

// the pages that the positions p0 .. p1 see together, in order: sink_pages from 0 on, then those from lo_page on, n in all (at least one)
struct Span {
    int sink_pages, lo_page, n;
    __device__ int page(int j) const { return j < sink_pages ? j : lo_page + (j - sink_pages); }
};
__device__ __forceinline__ int first_seen(const RowAttnArgs& a, int64_t p) {
    const int64_t lo = p - a.window + 1;
    return (int)min(max(lo, (int64_t)0), (int64_t)0x7fffffff);
}
__device__ __forceinline__ int last_seen(const RowAttnArgs& a, int64_t p) { return (int)min(p, (int64_t)a.max_blocks * kBlockSize - 1); }
__device__ __forceinline__ Span span_of(const RowAttnArgs& a, int64_t p0, int64_t p1) {
    Span s;
    const int end = last_seen(a, p1) / kBlockSize + 1;
    s.lo_page = min(first_seen(a, p0) / kBlockSize, end);
    s.sink_pages = min(a.n_sinks / kBlockSize + (a.n_sinks % kBlockSize != 0), s.lo_page);
    s.n = max(s.sink_pages + end - s.lo_page, 1);
    return s;
}

// the columns of a pass or a wave: tokens at the positions first .. last
struct Seen {
    int first_lo, last;                // first position in the window of the first token; last position that the last one sees
    int full_from, full_to, full_sinks;  // pages that every column sees all of: from .. to, and those below sinks
};
constexpr int kNoPage = 0x7fffffff;  // an entry that is no page: behind all of them
__device__ __forceinline__ Seen seen_of(const RowAttnArgs& a, int64_t p0, int64_t p1) {
    return Seen{first_seen(a, p0), last_seen(a, p1), first_seen(a, p1) / kBlockSize + (first_seen(a, p1) % kBlockSize != 0),
                (last_seen(a, p0) + 1) / kBlockSize - 1, a.n_sinks / kBlockSize};
}
__device__ __forceinline__ bool all_seen(const Seen& s, int page) { return (page <= s.full_to) & ((page >= s.full_from) | (page < s.full_sinks)); }
__device__ __forceinline__ bool sees(const RowAttnArgs& a, int lo, int last, int tok) {
    return (tok <= last) & ((tok >= lo) | (tok < a.n_sinks));
}

// masks of the bf16 pairs (0, 1) and (2, 3), or of the bytes, of the tokens tok .. tok+3 that some column sees
__device__ __forceinline__ uint4 seen_masks(const RowAttnArgs& a, const Seen& s, bool there, int tok) {
    bool v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = there && sees(a, s.first_lo, s.last, tok + r);
    const uint32_t bytes = (v[0] ? 0xffu : 0) | (v[1] ? 0xff00u : 0) | (v[2] ? 0xff0000u : 0) | (v[3] ? 0xff000000u : 0);
    return make_uint4((v[0] ? 0xffffu : 0) | (v[1] ? 0xffff0000u : 0), (v[2] ? 0xffffu : 0) | (v[3] ? 0xffff0000u : 0), bytes, 0);
}

// What a softmax's weights are relative to follows the running maximum only when that has grown by more than this many powers of two: weights
// and their sums stay below 2^8 times their number, in floating point as exact as below 1, and outputs are scaled once or twice a row.
constexpr float kSlack = 8.f;

// ---- operands ---------------------------------------------------------------------------------------------------

template <int FMT>
__host__ __device__ constexpr int pieces(int D) { return FMT == kFmtBf16 ? D / 32 : D / 64; }  // of 16 bytes per lane: a K or V tile
// the first of the 8 dims that a lane's operand of the 32 dims of step s holds
template <int FMT>
__device__ __forceinline__ int dim_of(int s, int lg) { return FMT == kFmtBf16 ? s * 32 + lg * 8 : s / 2 * 64 + lg * 16 + s % 2 * 8; }
template <int FMT, int N>
__device__ __forceinline__ bf16x8 key_operand(const uint4 (&k)[N], int s, float scale) {
    uint4 w;
    if (FMT == kFmtBf16) w = k[s % N];
    else {
        const uint4 c = k[s / 2];
        const uint2 a = widen8<FMT>(s % 2 ? c.z : c.x, scale), b = widen8<FMT>(s % 2 ? c.w : c.y, scale);
        w = make_uint4(a.x, a.y, b.x, b.y);
    }
    return *reinterpret_cast<bf16x8*>(&w);
}
// the largest of three, of four (of NaN and a number the number), without the instructions that the compiler puts before a maximum
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// A product that is rounded before it is added to another lane's.  Fused into the sum, a lane's own would enter unrounded and a + b and b + a differ: the
// term groups of a column would cut different weights into terms, and a weight near the end of a term lose 2^-16 of itself.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}
__device__ __forceinline__ uint32_t word(const uint4& w, int j) { return j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w; }
// An fp32 number is the sum of three bf16 terms, exactly: the first 8 of its 24 significant bits, the next 8 and the rest, by truncation.
// What is left of v behind its first t terms; its next term is the upper half of the word.
__device__ __forceinline__ float upper(float v, uint32_t mask) { return __uint_as_float(__float_as_uint(v) & mask); }
__device__ __forceinline__ float rest3(float v, int t) {
    const uint32_t m1 = t > 0 ? 0xffff0000u : 0, m2 = t > 1 ? 0xffff0000u : 0;
    const float r = v - upper(v, m1);
    return r - upper(r, m2);
}
__device__ __forceinline__ uint32_t uppers(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); }
// NaN and infinities among two bf16: the top bit of each half set where its exponent is all ones; as bf16 ones; and the word without them
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t ones_of(uint32_t bad) { return (bad >> 15) * 0x3f80u; }
__device__ __forceinline__ uint32_t without(uint32_t w, uint32_t bad) { return w & ~((bad >> 15) * 0xffffu); }
__device__ __forceinline__ uint4 finite_only(const uint4& w) {
    return make_uint4(without(w.x, not_finite(w.x)), without(w.y, not_finite(w.y)), without(w.z, not_finite(w.z)), without(w.w, not_finite(w.w)));
}

__device__ __forceinline__ intx4 mfma_i8(const uint4& a, const uint4& b, intx4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const intx4*>(&a), *reinterpret_cast<const intx4*>(&b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mfma32(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 mfma16(uint2 a, uint2 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(*reinterpret_cast<short4v*>(&a), *reinterpret_cast<short4v*>(&b), c, 0, 0, 0);
}

// Values that are no finite numbers, in a stage of pages of which a column sees some and another does not: 0 * NaN would reach those that do
// not see them.  The stage's products go on without them, and this, behind the loop over the stages, makes NaN of the dims and columns
// that have seen one: products of which values they are with which tokens a column sees.
template <int D, int NC, int NPG>
__device__ __forceinline__ void mark_not_finite(const RowAttnArgs& a, const Span& span, const Seen& seen, const int32_t* btrow, int c, int j0, int j1, const int (&col_lo)[NC],
                                                const int (&col_last)[NC], floatx4 (&o)[NC][D / 16]) {
    const int lane = threadIdx.x & 63, lg = lane >> 4;
    auto there = [&](int j, int& block) {
        const int page = j < j1 ? span.page(j) : kNoPage;
        block = page < a.max_blocks ? __builtin_amdgcn_readfirstlane(btrow[page]) : -1;
        return block < 0 || block >= a.num_blocks ? kNoPage : page;
    };
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
        int block;
        const int page = there(j, block), stage = j0 + (j - j0) / NPG * NPG;
        if (page == kNoPage) continue;
        bool full = true;
#pragma unroll 1
        for (int u = 0; u < NPG; ++u) {
            int other;
            full = full && all_seen(seen, there(stage + u, other));
        }
        if (full) continue;
        const int tok = page * kBlockSize + lg * 4;
        const uint4 keep = seen_masks(a, seen, true, tok);
        const uint8_t* tile = a.tiles + ((int64_t)block * a.n_kv + c) * (64 * D) + 32 * D + lane * 16;
        uint2 vis[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            uint32_t on[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) on[r] = sees(a, col_lo[n], col_last[n], tok + r) ? 0x3f80u : 0;
            vis[n] = make_uint2(on[0] | on[1] << 16, on[2] | on[3] << 16);
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(tile + i * 1024);
            const uint2 even = make_uint2(ones_of(not_finite(v.x & keep.x)), ones_of(not_finite(v.y & keep.y)));
            const uint2 odd = make_uint2(ones_of(not_finite(v.z & keep.x)), ones_of(not_finite(v.w & keep.y)));
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const floatx4 x = mfma16(even, vis[n], floatx4{0.f, 0.f, 0.f, 0.f}), y = mfma16(odd, vis[n], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    o[n][2 * i][r] = x[r] > 0.f ? NAN : o[n][2 * i][r];
                    o[n][2 * i + 1][r] = y[r] > 0.f ? NAN : o[n][2 * i + 1][r];
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// 16 bytes per lane from base + offset straight into LDS, as in device_util.h, with a scalar base
__device__ __forceinline__ void global_to_lds_16(const uint8_t* base, uint32_t offset, uint32_t lds_addr) {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory", "m0");
}

// a request's rows, as the kernels take them: 0 rows where the row starts do not ascend
struct Request {
    int r0, n;
    int64_t old;
};
__device__ __forceinline__ Request request(const RowAttnArgs& a, int i) {
    Request r;
    r.r0 = a.row_starts[i];
    const int r1 = a.row_starts[i + 1];
    r.n = r.r0 < 0 || r1 > a.rows || r1 <= r.r0 ? 0 : min(r1 - r.r0, a.max_new);
    r.old = max(a.seq_lens[i], 0);
    return r;
}

template <int D, bool F32>
__device__ __forceinline__ void store_row(const RowAttnArgs& a, int64_t row, int qhead, int e, floatx4 o) {
    const int64_t at = (row * a.n_kv * a.G + qhead) * D + e;
    if (F32) *reinterpret_cast<floatx4*>((float*)a.out + at) = o;
    else *reinterpret_cast<uint2*>((uint16_t*)a.out + at) = make_uint2(pack_bf16_rne(o[0], o[1]), pack_bf16_rne(o[2], o[3]));
}

// ---- requests of a few rows ---------------------------------------------------------------------------------------
// A pass: up to tg tokens of a request whose heads of one KV head fit the 16 columns; it reads the pages they see once, straight into operand
// registers.  The pages of all passes, one behind the other, are dealt out in equal shares to the waves of a KV head, whatever the requests'
// lengths: a wave finds its share from sums over the requests' lengths, 64 at a time, and may end one pass and begin others.  A pass
// that lies in several shares leaves partial results (maximum, sum, unnormalised output), which row_few_merge_kernel joins; partial result
// w + v is wave w's of pass v, a number of its own for each pair that exists.
//
// CW: columns of a term group.  Three terms of up to 4 columns share one instruction, of up to 8 two.  int8 keys meet the query in
// four 8-bit digits instead (whole multiples of 2^(f-24), with 2^f the power of two of the head's largest element: what is no smaller than
// 2^-7 of that is exact), on the 8-bit matrix cores: no key is widened, and sums are exact.
//
// Bound by memory where the caches are long: 32 requests of 24k to 32k tokens, 32 heads over 8 KV heads of 128, e4m3, fp32 queries 286 to 292 us, 6.5
// TB/s; over bf16 pages with a window of 4096 87 to 90 us, 6.1 TB/s.  One request of 8192 tokens takes 13 us and the join 4: launch, a chain of loads
// (row starts, table, page) and the partial results.  61 requests of up to 5000 tokens that bring up to 5, 16 heads over 2 of 64, e4m3: 27 us and 5.
//
// A share's least pages, us with 4 / 8 / 16: one request of 500 tokens 12.5 / 13.9 / 16.4, of 2000 13.6 / 14.4 / 17.0, of 8000 18.0 / 16.5 / 17.7, eight of 2000
// over bf16 pages 22.1 / 20.7 / 24.4: with fewer there are more partial results to join, with more the chain is longer.
constexpr int kFewMinPages = 8;
// Waves of a SIMD: two, but one where three terms of many columns and bf16 pages of 128 dims do not fit 256 registers.
__host__ __device__ constexpr int few_waves(int d, int fmt, bool f32, int cw, bool multi) {
    return fmt == kFmtBf16 && f32 && d == 128 && (cw == 16 || (cw == 8 && multi)) ? 1 : 2;
}
template <int D, int FMT, bool F32, int CW, bool MULTI>
__global__ __launch_bounds__(256, few_waves(D, FMT, F32, CW, MULTI)) void row_few_kernel(RowAttnArgs a) {
    constexpr bool DIGITS = FMT == kFmtInt8;
    constexpr int KSTEPS = D / (DIGITS ? 64 : 32), P = pieces<FMT>(D), NPG = D == 128 && (FMT == kFmtBf16 || (CW == 16 && (F32 || DIGITS))) ? 2 : 4;
    // terms of an instruction, and instructions, of a weight and of a query
    constexpr int TPP = F32 && CW <= 8 ? (CW <= 4 ? 3 : 2) : 1, NP = F32 ? (3 + TPP - 1) / TPP : 2;
    constexpr int TPQ = DIGITS ? 16 / CW : TPP, NQ = DIGITS ? 4 / TPQ : F32 ? NP : 1;
    constexpr float kDigits = TPQ == 1 ? 0x1p-8f : 0x1p-16f;  // from one instruction's digits to the next one's
    constexpr int TILE = FMT == kFmtBf16 ? 32 * D : 16 * D;               // bytes of a K or V tile
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_kv = a.n_kv, c = blockIdx.x % n_kv, w = blockIdx.x / n_kv * 4 + wave, W = gridDim.x / n_kv * 4;
    const int col = lane & 15, lg = lane >> 4, ci = col % CW, grp = col / CW;
    // columns behind the group's heads take the last one's place: what they load lies in q
    const int tq = MULTI ? ci / a.G : 0, h = MULTI ? ci - tq * a.G : min(ci, a.G - 1);

    // a lane's request of the 64 from i0 on, behind `before` passes: pages over its passes, and passes.  Requests whose passes have no record, of row starts
    // that do not ascend, are left out.
    auto look = [&](int i0, int before, Request& r, int& cost, int& np) {
        cost = np = 0;
        if (i0 + lane < a.batch) {
            r = request(a, i0 + lane);
            if (r.n > 0 && r.n <= a.few_max) {
                np = (r.n + a.tg - 1) / a.tg;
                for (int g = 0; g < np; ++g) cost += span_of(a, r.old + g * a.tg, r.old + min((g + 1) * a.tg, r.n) - 1).n;
            }
        }
        if (before + wave_scan(np) > a.passes_max) cost = np = 0;
    };
    int64_t total = 0;
    int n_pass = 0;
    Request rq;
    int cost, np;
    for (int i0 = 0; i0 < a.batch; i0 += 64) {
        look(i0, n_pass, rq, cost, np);
        total += wave_total(cost);
        n_pass += wave_total(np);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) a.head[0] = n_pass;
    int64_t share64 = max((total + W - 1) / W, (int64_t)kFewMinPages);
    const int share = (int)((share64 + NPG - 1) / NPG * NPG);
    const int64_t begin = (int64_t)w * share, end = min(begin + share, total);
    if (begin >= end) return;

    int64_t base = 0, at = begin;
    int vbase = 0;
    for (int i0 = 0; i0 < a.batch && at < end; i0 += 64) {
        if (a.batch > 64) look(i0, vbase, rq, cost, np);  // else they are still there
        const int incl = wave_scan(cost), vincl = wave_scan(np);
        const int all = __builtin_amdgcn_readlane(incl, 63);
        uint64_t ahead = __ballot(base + incl > at && cost > 0);
        while (ahead && at < end) {
            const int L = __builtin_ctzll(ahead);
            ahead &= ahead - 1;
            const int row0 = __builtin_amdgcn_readlane(rq.r0, L), n = __builtin_amdgcn_readlane(rq.n, L);
            const int64_t old = __builtin_amdgcn_readlane((int)rq.old, L);
            const int passes = __builtin_amdgcn_readlane(np, L);
            int64_t first = base + __builtin_amdgcn_readlane(incl, L) - __builtin_amdgcn_readlane(cost, L);
            int v = vbase + __builtin_amdgcn_readlane(vincl, L) - passes;
            for (int g = 0; g < passes && at < end; ++g, ++v) {
                const int t0 = g * a.tg, tv = MULTI ? min(a.tg, n - t0) : 1;
                const Span span = span_of(a, old + t0, old + t0 + tv - 1);
                const int64_t pass0 = first;
                first += span.n;
                if (first <= at) continue;
                const int j0 = (int)(at - pass0), j1 = (int)min((int64_t)span.n, end - pass0);
                at = pass0 + j1;
                const int seg0 = (int)(pass0 / share), segs = (int)((first - 1) / share) - seg0 + 1;
                if (j0 == 0 && c == 0 && lane == 0)
                    *reinterpret_cast<int4*>(a.head + 4 + 4 * (size_t)v) = make_int4(row0 + t0, tv, seg0 + v, segs);

                // ---- the pages j0 .. j1-1 of pass v
                const bool on = ci < a.G * tv;
                const Seen seen = seen_of(a, old + t0, old + t0 + tv - 1);
                const int64_t pos = old + t0 + min(tq, tv - 1);
                const int lo1[1] = {first_seen(a, pos)}, last1[1] = {last_seen(a, pos)};
                const int32_t* btrow = a.bt + (size_t)(i0 + L) * a.max_blocks;

                // lane l holds entry lbase + l of the span: the page, where it is in the pool, its powers of two
                int lbase = j0, v_page, v_block, v_exp = 0;
                auto fetch = [&] {
                    const int j = lbase + lane;
                    int pg = j < j1 ? span.page(j) : kNoPage, blk = -1;
                    if (pg < a.max_blocks) blk = btrow[pg];
                    if (blk < 0 || blk >= a.num_blocks) pg = kNoPage, blk = 0;  // nothing there: page 0 of the pool is read and masked
                    v_page = pg;
                    v_block = blk;
                    if (FMT != kFmtBf16) v_exp = *reinterpret_cast<const uint16_t*>(a.exps + ((int64_t)blk * n_kv + c) * 2);
                };
                struct Stage {
                    uint4 k[NPG][P], v[NPG][P];
                    int page[NPG];
                } cur, nxt;
                auto load = [&](int j, Stage& s) {
                    if (j - lbase >= 64) {  // uniform; 64 is a multiple of NPG
                        lbase = j;
                        fetch();
                    }
#pragma unroll
                    for (int u = 0; u < NPG; ++u) {
                        const bool there = j + u < j1;
                        const int l = (j + u - lbase) & 63;
                        s.page[u] = there ? __builtin_amdgcn_readlane(v_page, l) : kNoPage;
                        const int blk = there ? __builtin_amdgcn_readlane(v_block, l) : 0;
                        const uint8_t* tile = a.tiles + ((int64_t)blk * n_kv + c) * (2 * TILE) + lane * 16;
#pragma unroll
                        for (int i = 0; i < P; ++i) {
                            s.k[u][i] = load_stream_16(tile + i * 1024);
                            s.v[u][i] = load_stream_16(tile + TILE + i * 1024);
                        }
                    }
                };
                uint4 qt[NQ][KSTEPS];
                float qw = 0.f;  // what a digit of the lane's first term stands for
                floatx4 oo[1][D / 16], (&o)[D / 16] = oo[0];
#pragma unroll
                for (int t = 0; t < D / 16; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
                float m_ref = -INFINITY, l_run = 0.f;
                bool marked = false;

                fetch();
                load(j0, cur);
                __builtin_amdgcn_sched_barrier(0);
                const int64_t qrow = (row0 + t0 + min(tq, tv - 1)) * a.q_stride + (int64_t)(c * a.G + h) * D;
                if (DIGITS) {
                    float y[KSTEPS][16], top = 0.f;
                    bool odd = false;
#pragma unroll
                    for (int s = 0; s < KSTEPS; ++s) {
                        const int64_t at = qrow + s * 64 + lg * 16;
#pragma unroll
                        for (int e = 0; e < 16; e += 4) {
                            if (F32) {
                                const float4 z = *reinterpret_cast<const float4*>((const float*)a.q + at + e);
                                y[s][e] = z.x, y[s][e + 1] = z.y, y[s][e + 2] = z.z, y[s][e + 3] = z.w;
                            } else {
                                const uint2 z = *reinterpret_cast<const uint2*>((const uint16_t*)a.q + at + e);
                                y[s][e] = bf16_lo(z.x), y[s][e + 1] = bf16_hi(z.x), y[s][e + 2] = bf16_lo(z.y), y[s][e + 3] = bf16_hi(z.y);
                            }
#pragma unroll
                            for (int z = 0; z < 4; ++z) {
                                top = fmaxf(top, fabsf(y[s][e + z]));
                                odd |= !(fabsf(y[s][e + z]) < INFINITY);
                            }
                        }
                    }
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    // |y| <= 127 * 2^f; a head of zeros, NaN and infinities go by any power (the last two are put back below)
                    const int f = top > 0.f && top < INFINITY ? max(power_of(top), -100) : 0;
                    const float up = two_to(-f) * 0x1p24f;
#pragma unroll
                    for (int s = 0; s < KSTEPS; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t w[4] = {0, 0, 0, 0};  // four elements' digits, high ones first
#pragma unroll
                            for (int z = 0; z < 4; ++z) {
                                const int x = on ? (int)rintf(y[s][4 * e + z] * up) : 0;
                                // low digit first, each -128 .. 127: |x| <= 127 * 2^24 leaves -127 .. 127 for the high one
                                const int d3 = (int8_t)x, x2 = (x - d3) >> 8, d2 = (int8_t)x2, x1 = (x2 - d2) >> 8, d1 = (int8_t)x1, d0 = (x1 - d1) >> 8;
                                w[0] |= (uint32_t)(d0 & 0xff) << (8 * z);
                                w[1] |= (uint32_t)(d1 & 0xff) << (8 * z);
                                w[2] |= (uint32_t)(d2 & 0xff) << (8 * z);
                                w[3] |= (uint32_t)(d3 & 0xff) << (8 * z);
                            }
#pragma unroll
                            for (int i = 0; i < NQ; ++i) {
                                const int t = i * TPQ + grp;
                                const uint32_t v = t == 0 ? w[0] : t == 1 ? w[1] : t == 2 ? w[2] : w[3];
                                if (e == 0) qt[i][s].x = v;
                                else if (e == 1) qt[i][s].y = v;
                                else if (e == 2) qt[i][s].z = v;
                                else qt[i][s].w = v;
                            }
                        }
                    float bad = odd ? NAN : 0.f;
                    bad += __shfl_xor(bad, 16);
                    bad += __shfl_xor(bad, 32);
                    qw = two_to(f) * a.scale_log2e * two_to(-8 * grp) + (on ? bad : 0.f);
                } else {
#pragma unroll
                    for (int s = 0; s < KSTEPS; ++s) {
                        const int64_t at = qrow + dim_of<FMT>(s, lg);
                        if (F32) {
                            const float4 y0 = *reinterpret_cast<const float4*>((const float*)a.q + at), y1 = *reinterpret_cast<const float4*>((const float*)a.q + at + 4);
                            const float y[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
                            for (int i = 0; i < NQ; ++i) {
                                float z[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const int t = i * TPP + grp;
                                    z[e] = !on || grp >= TPP || t > 2 ? 0.f : rest3(y[e] * a.scale_log2e, t);
                                }
                                qt[i][s] = make_uint4(uppers(z[0], z[1]), uppers(z[2], z[3]), uppers(z[4], z[5]), uppers(z[6], z[7]));
                            }
                        } else {
                            const uint4 y = *reinterpret_cast<const uint4*>((const uint16_t*)a.q + at);
                            qt[0][s] = on ? y : make_uint4(0, 0, 0, 0);
                        }
                    }
                }

                for (int j = j0; j < j1; j += NPG) {
                    // the powers of two that load() may overwrite; taken here, no page's load waits for them
                    int exps[NPG];
#pragma unroll
                    for (int u = 0; u < NPG; ++u) exps[u] = FMT == kFmtBf16 || j + u >= j1 ? 0 : __builtin_amdgcn_readlane(v_exp, (j + u - lbase) & 63);
                    if (j + NPG < j1) load(j + NPG, nxt);
                    __builtin_amdgcn_sched_barrier(0);
                    bool full = true;
#pragma unroll
                    for (int u = 0; u < NPG; ++u) full &= all_seen(seen, cur.page[u]);
                    floatx4 x[NPG];
                    float ks[NPG], vs[NPG];
#pragma unroll
                    for (int u = 0; u < NPG; ++u) {
                        ks[u] = FMT == kFmtBf16 ? 1.f : two_to((int8_t)(exps[u] & 0xff));
                        vs[u] = FMT == kFmtBf16 ? 1.f : two_to((int8_t)(exps[u] >> 8));
                        if (DIGITS) {
                            intx4 y[NQ];
#pragma unroll
                            for (int i = 0; i < NQ; ++i) {
                                y[i] = intx4{0, 0, 0, 0};
#pragma unroll
                                for (int k = 0; k < KSTEPS; ++k) y[i] = mfma_i8(cur.k[u][k % P], qt[i][k], y[i]);
                            }
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                float v = (float)y[NQ - 1][r];
#pragma unroll
                                for (int i = NQ - 2; i >= 0; --i) v = fmaf(v, kDigits, (float)y[i][r]);
                                x[u][r] = rounded_product(v, qw * ks[u]);  // every group adds the same numbers below
                            }
                        } else {
                            x[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int k = 0; k < KSTEPS; ++k) {
                                const bf16x8 key = key_operand<FMT>(cur.k[u], k, ks[u]);
#pragma unroll
                                for (int i = 0; i < NQ; ++i) x[u] = mfma32(key, *reinterpret_cast<bf16x8*>(&qt[i][k]), x[u]);
                            }
                            if (!F32) x[u] *= a.scale_log2e;
                        }
                        if (TPQ > 1) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) {  // the sum over the term groups, in every column
                                x[u][r] += row_move<kRor8>(x[u][r]);
                                if (CW <= 4) x[u][r] += row_move<kRor4>(x[u][r]);
                            }
                        }
                    }
                    if (!full) {
#pragma unroll
                        for (int u = 0; u < NPG; ++u) {
                            const bool there = cur.page[u] != kNoPage;
                            const int tok = (there ? cur.page[u] : 0) * kBlockSize + lg * 4;
                            if (!there) vs[u] = 0.f;
#pragma unroll
                            for (int r = 0; r < 4; ++r) x[u][r] = there && sees(a, lo1[0], last1[0], tok + r) ? x[u][r] : -INFINITY;
                            // what no column sees may hold anything, NaN included: clear its V so that 0 * V stays 0
                            const uint4 keep = seen_masks(a, seen, there, tok);
#pragma unroll
                            for (int i = 0; i < P; ++i) {
                                uint4& v = cur.v[u][i];
                                if (FMT == kFmtBf16) v.x &= keep.x, v.y &= keep.y, v.z &= keep.x, v.w &= keep.y;
                                else v.x &= keep.z, v.y &= keep.z, v.z &= keep.z, v.w &= keep.z;
                            }
                        }
                        if (FMT == kFmtBf16 && MULTI) {  // 8-bit caches hold none
                            uint32_t bad = 0;
#pragma unroll
                            for (int u = 0; u < NPG; ++u)
#pragma unroll
                                for (int i = 0; i < P; ++i) {
                                    const uint4 v = cur.v[u][i];
                                    bad |= not_finite(v.x) | not_finite(v.y) | not_finite(v.z) | not_finite(v.w);
                                }
                            if (__any(bad != 0)) {
                                marked = true;
#pragma unroll
                                for (int u = 0; u < NPG; ++u)
#pragma unroll
                                    for (int i = 0; i < P; ++i) cur.v[u][i] = finite_only(cur.v[u][i]);
                            }
                        }
                    }
                    float mx = x[0][0];
#pragma unroll
                    for (int u = 0; u < NPG; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[u][r]);
                    const bool grown = __any(mx > m_ref + kSlack);
                    float alpha = 1.f;
                    if (grown) {
                        mx = fmaxf(mx, __shfl_xor(mx, 16));
                        mx = fmaxf(mx, __shfl_xor(mx, 32));
                        const float m_new = fmaxf(m_ref, mx);
                        alpha = __builtin_amdgcn_exp2f(m_ref - fmaxf(m_new, -1e30f));
                        m_ref = m_new;
                        l_run *= alpha;
                    }
#pragma unroll
                    for (int t = 0; t < D / 16; t += 4) {  // four blocks to a branch: the compiler holds what a branch changes twice
                        if (grown) {
#pragma unroll
                            for (int z = 0; z < 4; ++z) o[t + z] *= alpha;
                        }
                        asm volatile("");
                    }
                    const float m_use = fmaxf(m_ref, -1e30f);  // nothing seen yet: finite exponents, weights 0
#pragma unroll
                    for (int u = 0; u < NPG; u += 2) {
                        float pr[2][4];
#pragma unroll
                        for (int z = 0; z < 2; ++z)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                pr[z][r] = __builtin_amdgcn_exp2f(x[u + z][r] - m_use);
                                l_run += pr[z][r];
                                if (DIGITS) pr[z][r] *= vs[u + z];  // int8 values enter as their codes
                            }
                        uint4 pt[NP];
#pragma unroll
                        for (int i = 0; i < NP; ++i) {
                            // with bf16 queries two terms, 16 bits: one of 8 would add as much error as out's own rounding where a row has few columns
                            const int t = TPP > 1 ? i * TPP + grp : i;
                            const uint32_t keep = TPP > 1 && (t > 2 || grp >= TPP) ? 0 : ~0u;
                            float y[2][4];
#pragma unroll
                            for (int z = 0; z < 2; ++z)
#pragma unroll
                                for (int r = 0; r < 4; ++r) y[z][r] = rest3(pr[z][r], t);
                            pt[i] = make_uint4(uppers(y[0][0], y[0][1]) & keep, uppers(y[0][2], y[0][3]) & keep, uppers(y[1][0], y[1][1]) & keep,
                                               uppers(y[1][2], y[1][3]) & keep);
                        }
#pragma unroll
                        for (int b = 0; b < D / 16; ++b) {
                            if (FMT == kFmtBf16) {
                                const uint4 &va = cur.v[u][b / 2 % P], &vb = cur.v[u + 1][b / 2 % P];
                                const uint2 v0 = b % 2 ? make_uint2(va.z, va.w) : make_uint2(va.x, va.y);
                                const uint2 v1 = b % 2 ? make_uint2(vb.z, vb.w) : make_uint2(vb.x, vb.y);
#pragma unroll
                                for (int i = 0; i < NP; ++i) {
                                    o[b] = mfma16(v0, make_uint2(pt[i].x, pt[i].y), o[b]);
                                    o[b] = mfma16(v1, make_uint2(pt[i].z, pt[i].w), o[b]);
                                }
                            } else {
                                const float s0 = DIGITS ? 1.f : vs[u], s1 = DIGITS ? 1.f : vs[u + 1];
                                const uint2 v0 = widen8<FMT>(word(cur.v[u][b / 4 % P], b % 4), s0), v1 = widen8<FMT>(word(cur.v[u + 1][b / 4 % P], b % 4), s1);
                                uint4 v = make_uint4(v0.x, v0.y, v1.x, v1.y);
#pragma unroll
                                for (int i = 0; i < NP; ++i) o[b] = mfma32(*reinterpret_cast<bf16x8*>(&v), *reinterpret_cast<bf16x8*>(&pt[i]), o[b]);
                            }
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    cur = nxt;
                }

                if (FMT == kFmtBf16 && MULTI && marked) mark_not_finite<D, 1, NPG>(a, span, seen, btrow, c, j0, j1, lo1, last1, oo);
                l_run += __shfl_xor(l_run, 16);
                l_run += __shfl_xor(l_run, 32);
                if (TPP > 1 && F32) {
#pragma unroll
                    for (int t = 0; t < D / 16; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            o[t][r] += row_move<kRor8>(o[t][r]);
                            if (CW <= 4) o[t][r] += row_move<kRor4>(o[t][r]);
                        }
                }
                if (grp == 0 && on) {
                    if (segs == 1) {
                        const float by = 1.f / (l_run > 0.f || l_run != l_run ? l_run : 1.f);
#pragma unroll
                        for (int t = 0; t < D / 16; ++t)
                            store_row<D, F32>(a, row0 + t0 + tq, c * a.G + h, t * 16 + lg * 4, o[t] * by);
                    } else {
                        const int64_t slot = ((int64_t)(w + v) * n_kv + c) * a.pcols + ci;
                        if (lg == 0) {
                            a.part_ml[slot * 2] = fmaxf(m_ref, -1e30f);
                            a.part_ml[slot * 2 + 1] = l_run;
                        }
#pragma unroll
                        for (int t = 0; t < D / 16; ++t) *reinterpret_cast<floatx4*>(a.part_o + slot * D + t * 16 + lg * 4) = o[t];
                    }
                }
            }
        }
        base += all;
        vbase += __builtin_amdgcn_readlane(vincl, 63);
    }
}

// joins the partial results of a pass: a workgroup per (pass, KV head, column), in slices of 32 (D = 128) or 16 lanes, in a fixed order
template <int D, bool F32>
__global__ __launch_bounds__(256) void row_few_merge_kernel(RowAttnArgs a) {
    constexpr int LANES = D / 4, S = 256 / LANES;
    __shared__ floatx4 s_num[S][LANES];
    __shared__ float s_den[S], s_max[S];
    const int col = blockIdx.x % a.pcols, vc = blockIdx.x / a.pcols, c = vc % a.n_kv, v = vc / a.n_kv;
    const int n_pass = a.head[0];
    const int4 rec = *reinterpret_cast<const int4*>(a.head + 4 + 4 * (size_t)v);  // asked for beside the count; behind it whatever lies there
    if (v >= n_pass || rec.w <= 1 || col >= a.G * rec.y) return;
    const int sl = threadIdx.x / LANES, ln = threadIdx.x % LANES;
    float M = -1e30f, den = 0.f;
    floatx4 num = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAtOnce = 4;  // parts whose loads are on their way together
    for (int j0 = sl; j0 < rec.w; j0 += S * kAtOnce) {
        float2 ml[kAtOnce];
        floatx4 o[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t slot = ((int64_t)(rec.z + min(j0 + u * S, rec.w - 1)) * a.n_kv + c) * a.pcols + col;
            ml[u] = *reinterpret_cast<const float2*>(a.part_ml + slot * 2);
            o[u] = *reinterpret_cast<const floatx4*>(a.part_o + slot * D + ln * 4);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (j0 + u * S < rec.w) {
                const float Mn = fmaxf(M, ml[u].x), f0 = __builtin_amdgcn_exp2f(M - Mn), f1 = __builtin_amdgcn_exp2f(ml[u].x - Mn);
                num = num * f0 + o[u] * f1;
                den = den * f0 + ml[u].y * f1;
                M = Mn;
            }
    }
    s_num[sl][ln] = num;
    if (ln == 0) {
        s_den[sl] = den;
        s_max[sl] = M;
    }
    __syncthreads();
    if (sl != 0) return;
#pragma unroll
    for (int j = 1; j < S; ++j) M = fmaxf(M, s_max[j]);
    num = floatx4{0.f, 0.f, 0.f, 0.f};
    den = 0.f;
#pragma unroll
    for (int j = 0; j < S; ++j) {
        const float f = __builtin_amdgcn_exp2f(s_max[j] - M);
        num += s_num[j][ln] * f;
        den += s_den[j] * f;
    }
    const int tq = col / a.G, h = col - tq * a.G;
    if (!(den > 0.f) && den == den) den = 1.f;
    store_row<D, F32>(a, (int64_t)rec.x + tq, c * a.G + h, ln * 4, num * (1.f / den));
}

// ---- requests of many rows ----------------------------------------------------------------------------------------
// A workgroup takes a tile of tt tokens x G heads of one KV head, up to 128 columns, 32 of them a wave's, and goes through the pages
// that they see together in stages of two: the next stage's come into LDS, as bf16 in operand order, while this one's are multiplied.
// A column group's maxima, sums and outputs stay in registers.  Tiles with the most pages begin first.  Where there are few tiles
// the pages of each are dealt to `splits` workgroups.
//
// Bound by the latency of a stage (barrier, LDS reads, the softmax between two products) and the vector units more than by the matrix cores, which
// are busy 32 % of the time (vector units 40 to 50 %): a prompt of 8192 tokens within a window of 1024, 32 heads over 8 KV heads of 128, bf16 181 us a call
// among others, 0.71 PFLOP/s of the 1.41 that a large product reaches here; three chunks of 500 to 1100 tokens behind 12k tokens of int8 pages 581 to 607 us, 0.8 PFLOP/s.  Two pages
// a stage leave registers and LDS for three waves of a SIMD: the chunks 617 us, and 803 with four pages and two waves.  Splitting the chunks' pages 609 us,
// not splitting them 666; 29 mixed requests in fp32 within a window of 777 75.1 and 78.7.
constexpr int kManyTiles = 2, kManyCols = 64 * kManyTiles;  // column tiles of a wave; columns of a workgroup
struct ManyTile {
    int r0, t0, tv, req;
    int64_t old;
};
// Which tile a slot is, by a whole wave: of the requests of more than few_max rows the k-th owns the slots from row_starts/tt + k on.  Its tiles end before
// the next one's begin (x/tt + n/tt rounded up is at most (x+n)/tt + 1), and there are no more of them than rows/(few_max+1), so that neither requests of few
// rows nor those without rows take a slot.
__device__ __forceinline__ bool many_tile(const RowAttnArgs& a, int slot, ManyTile& m) {
    const int lane = threadIdx.x & 63;
    int before = 0, local = -1;
    for (int i0 = 0; i0 < a.batch; i0 += 64) {
        Request r = request(a, min(i0 + lane, a.batch - 1));
        const bool many = i0 + lane < a.batch && r.n > a.few_max;
        const uint64_t all = __ballot(many);
        const int at = r.r0 / a.tt + before + __popcll(all & (((uint64_t)1 << lane) - 1));
        const uint64_t begun = __ballot(many && at <= slot);
        if (begun) {  // the last of them
            const int L = 63 - __builtin_clzll(begun);
            m.req = i0 + L;
            m.r0 = __builtin_amdgcn_readlane(r.r0, L);
            m.tv = __builtin_amdgcn_readlane(r.n, L);
            m.old = __builtin_amdgcn_readlane((int)r.old, L);
            local = slot - __builtin_amdgcn_readlane(at, L);
        }
        if (begun != all) break;
        before += __popcll(all);
    }
    if (local < 0) return false;
    const int tiles = (m.tv + a.tt - 1) / a.tt;
    if (local >= tiles) return false;
    m.t0 = (tiles - 1 - local) * a.tt;  // the last tokens see the most
    m.tv = min(a.tt, m.tv - m.t0);
    return true;
}

template <int D, int FMT, bool F32>
__global__ __launch_bounds__(256, F32 ? 2 : 3) void row_many_kernel(RowAttnArgs a) {
    constexpr int KSTEPS = D / 32, P = pieces<FMT>(D), NB = D / 16, NC = kManyTiles, NT = F32 ? 3 : 1;
    constexpr int TILE = FMT == kFmtBf16 ? 32 * D : 16 * D;
    // What a wave brings of a stage: pieces of K (KEYS of them), and of V a piece (bf16) or half of one (8 bits) of both pages
    constexpr int KEYS = (2 * P + 3) / 4, VALUES = FMT == kFmtBf16 ? P : 2 * P;
    __shared__ uint4 s_k[2][2][KSTEPS][64];  // [buffer][page][step][lane]
    __shared__ uint4 s_v[2][NB][64];         // [buffer][16 dims][lane]: 4 tokens of either page
    __shared__ int s_marked;                 // some value was no finite number
    if (threadIdx.x == 0) s_marked = 0;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_kv = a.n_kv, c = blockIdx.x % n_kv, rest = blockIdx.x / n_kv, split = rest % a.splits, slot = rest / a.splits;
    const int col = lane & 15, lg = lane >> 4;
    ManyTile m;
    if (!many_tile(a, slot, m)) return;
    const int live = a.G * m.tv;
    const Span span = span_of(a, m.old + m.t0, m.old + m.t0 + m.tv - 1);
    const Seen tile_seen = seen_of(a, m.old + m.t0, m.old + m.t0 + m.tv - 1);
    const int stages = (span.n + 1) / 2, st0 = (int)((int64_t)stages * split / a.splits), st1 = (int)((int64_t)stages * (split + 1) / a.splits);
    const int32_t* btrow = a.bt + (size_t)m.req * a.max_blocks;

    // the wave's columns
    const int wc = wave * 16 * NC;
    const bool idle = wc >= live;
    const int64_t pw = m.old + m.t0;
    const Seen seen = seen_of(a, pw + min(wc / a.G, m.tv - 1), pw + min((wc + 16 * NC - 1) / a.G, m.tv - 1));
    int col_lo[NC], col_last[NC];
    uint4 qt[NC][NT][KSTEPS];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        const int ci = wc + n * 16 + col, tq = min(ci / a.G, m.tv - 1), h = ci % a.G;
        col_lo[n] = first_seen(a, pw + tq);
        col_last[n] = last_seen(a, pw + tq);
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            // 8-bit keys lie in LDS as the bf16 pool's do, step for step
            const int64_t qat = (int64_t)(m.r0 + m.t0 + tq) * a.q_stride + (int64_t)(c * a.G + h) * D + dim_of<FMT>(s, lg);
            if (F32) {
                const float* qp = (const float*)a.q + qat;
                const float4 y0 = *reinterpret_cast<const float4*>(qp), y1 = *reinterpret_cast<const float4*>(qp + 4);
                const float y[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    float z[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = ci < live ? rest3(y[e] * a.scale_log2e, i) : 0.f;
                    qt[n][i][s] = make_uint4(uppers(z[0], z[1]), uppers(z[2], z[3]), uppers(z[4], z[5]), uppers(z[6], z[7]));
                }
            } else {
                const uint4 y = *reinterpret_cast<const uint4*>((const uint16_t*)a.q + qat);
                qt[n][0][s] = ci < live ? y : make_uint4(0, 0, 0, 0);
            }
        }
    }
    floatx4 o[NC][NB];
    float m_ref[NC];
    floatx4 l_run[NC];  // fp32: the lane's own tokens' sum in [0]; bf16: all tokens', of the rounded weights, by a product with ones
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        m_ref[n] = -INFINITY;
        l_run[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < NB; ++b) o[n][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    // lane l holds entry lbase + l of the span
    int lbase = st0 * 2, v_page, v_block, v_exp = 0;
    auto fetch = [&] {
        const int j = lbase + lane;
        int pg = j < span.n ? span.page(j) : kNoPage, blk = -1;
        if (pg < a.max_blocks) blk = btrow[pg];
        if (blk < 0 || blk >= a.num_blocks) pg = kNoPage, blk = 0;
        v_page = pg;
        v_block = blk;
        if (FMT != kFmtBf16) {
            v_exp = *reinterpret_cast<const uint16_t*>(a.exps + ((int64_t)blk * n_kv + c) * 2);
            if (pg == kNoPage) v_exp = 0;  // whatever page 0 has: its values are cleared
        }
    };
    u32x4 rk[FMT == kFmtBf16 ? 1 : KEYS], rv[2];  // what the wave brings of the stage that comes next
    int exps[2] = {0, 0}, cur_exps[2], pages[2], next_pages[2];
    const int v_unit = wave - (4 - VALUES);  // below 0: no V
    const uint32_t lane16 = lane * 16u;      // beside a scalar base
    auto load = [&](int st, int buf) {
        if (st * 2 - lbase >= 64) {
            lbase = st * 2;
            fetch();
        }
        const int l = st * 2 - lbase;  // 2 divides 64
        const uint8_t* tile[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            next_pages[u] = __builtin_amdgcn_readlane(v_page, l + u);
            exps[u] = __builtin_amdgcn_readlane(v_exp, l + u);
            tile[u] = a.tiles + ((int64_t)__builtin_amdgcn_readlane(v_block, l + u) * n_kv + c) * (2 * TILE);
        }
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int k = wave * KEYS + i, page = k / P, piece = k % P;
            if (k < 2 * P) {  // uniform
                const uint8_t* src = (page ? tile[1] : tile[0]) + piece * 1024;
                if (FMT == kFmtBf16) global_to_lds_16(src, lane16, lds_address(&s_k[buf][page][piece][0]));
                else rk[i] = *reinterpret_cast<const u32x4*>(src + lane16);
            }
        }
        if (v_unit >= 0) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t* src = tile[u] + TILE;
                if (FMT == kFmtBf16) rv[u] = *reinterpret_cast<const u32x4*>(src + v_unit * 1024 + lane16);
                else {
                    const uint2 half = *reinterpret_cast<const uint2*>(src + (v_unit / 2 * 1024 + v_unit % 2 * 8) + lane16);
                    rv[u][0] = half.x;
                    rv[u][1] = half.y;
                }
            }
        }
    };
    auto put = [&](int buf) {
        if (FMT != kFmtBf16) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const int k = wave * KEYS + i, page = k / P, piece = k % P;
                if (k < 2 * P) {
                    const float ks = FMT == kFmtE4m3 ? two_to((int8_t)((page ? exps[1] : exps[0]) & 0xff)) : 1.f;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const uint2 x = widen8<FMT>(rk[i][2 * s], ks), y = widen8<FMT>(rk[i][2 * s + 1], ks);
                        s_k[buf][page][2 * piece + s][lane] = make_uint4(x.x, x.y, y.x, y.y);
                    }
                }
            }
        }
        if (v_unit < 0) return;
        float vs[2] = {1.f, 1.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (FMT == kFmtE4m3) vs[u] = two_to((int8_t)(exps[u] >> 8));
            if (!all_seen(tile_seen, next_pages[u])) {  // what no column of the tile sees may hold anything
                const bool there = next_pages[u] != kNoPage;
                const uint4 keep = seen_masks(a, tile_seen, there, (there ? next_pages[u] : 0) * kBlockSize + lg * 4);
                rv[u] &= FMT == kFmtBf16 ? u32x4{keep.x, keep.y, keep.x, keep.y} : u32x4{keep.z, keep.z, keep.z, keep.z};
                if (FMT == kFmtBf16) {
                    const uint32_t bad = not_finite(rv[u][0]) | not_finite(rv[u][1]) | not_finite(rv[u][2]) | not_finite(rv[u][3]);
                    if (__any(bad != 0)) {
                        s_marked = 1;
#pragma unroll
                        for (int e = 0; e < 4; ++e) rv[u][e] = without(rv[u][e], not_finite(rv[u][e]));
                    }
                }
            }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {  // two blocks of 16 dims
            if (FMT == kFmtBf16) s_v[buf][2 * v_unit + b][lane] = make_uint4(rv[0][2 * b], rv[0][2 * b + 1], rv[1][2 * b], rv[1][2 * b + 1]);
            else {
                const uint2 x = widen8<FMT>(rv[0][b], vs[0]), y = widen8<FMT>(rv[1][b], vs[1]);
                s_v[buf][2 * v_unit + b][lane] = make_uint4(x.x, x.y, y.x, y.y);
            }
        }
    };

    auto compute = [&](int buf) {
        if (idle) return;
        // int8 codes are multiplied as they are: the keys' power of two goes to the scores, the values' to the weights.  fp32 rows' weights are added up before.  Those
        // of bf16 rows get it within the exponential, and the product that adds them up takes it out: a page of zeros, whose power is 2^-100, so loses its weights
        // below 2^-26 (of a sum of at least 1), no more than that sum does, which is off by up to 2^-24 for each.
        constexpr bool INT8 = FMT == kFmtInt8, SCALED = INT8 || !F32, FOLDED = INT8 && !F32;
        float ks[2], ev[2], vup[2];
        uint32_t one[2] = {0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            ks[u] = F32 ? 1.f : a.scale_log2e;
            if (INT8) {
                const int e = (int8_t)(cur_exps[u] >> 8);
                ks[u] *= two_to((int8_t)(cur_exps[u] & 0xff));
                ev[u] = (float)e;
                vup[u] = two_to(e);
                one[u] = (uint32_t)(127 - e) << 23 | (uint32_t)(127 - e) << 7;
            }
        }
        floatx4 x[NC][2];
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint4 kw = s_k[buf][u][s][lane];
#pragma unroll
                for (int n = 0; n < NC; ++n)
#pragma unroll
                    for (int i = 0; i < NT; ++i)
                        x[n][u] = mfma32(*reinterpret_cast<bf16x8*>(&kw), *reinterpret_cast<bf16x8*>(&qt[n][i][s]),
                                         s == 0 && i == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : x[n][u]);
            }
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (!all_seen(seen, pages[u])) {
                const bool there = pages[u] != kNoPage;
                const int tok = (there ? pages[u] : 0) * kBlockSize + lg * 4;
#pragma unroll
                for (int n = 0; n < NC; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[n][u][r] = there && sees(a, col_lo[n], col_last[n], tok + r) ? x[n][u][r] : -INFINITY;
            }
        float top[NC];
        bool above = false;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const floatx4 y = x[n][0], z = x[n][1];
            if (INT8) top[n] = fmaxf(max3(max3(y[0], y[1], y[2]), y[3], y[3]) * ks[0], max3(max3(z[0], z[1], z[2]), z[3], z[3]) * ks[1]);
            else {
                top[n] = max3(max3(max3(y[0], y[1], y[2]), y[3], z[0]), max3(z[1], z[2], z[3]), -INFINITY);
                if (SCALED) top[n] *= a.scale_log2e;
            }
            above |= top[n] > m_ref[n] + kSlack;
        }
        const bool grown = __any(above);
        float alpha[NC];
        if (grown) {
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                top[n] = fmaxf(top[n], __shfl_xor(top[n], 16));
                top[n] = fmaxf(top[n], __shfl_xor(top[n], 32));
                const float m_new = fmaxf(m_ref[n], top[n]);
                alpha[n] = __builtin_amdgcn_exp2f(m_ref[n] - fmaxf(m_new, -1e30f));
                m_ref[n] = m_new;
                l_run[n] *= alpha[n];
            }
        }
        // four blocks to a branch: the compiler holds what a branch changes twice
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int b = 0; b < NB; b += 4) {
                if (grown) {
#pragma unroll
                    for (int z = 0; z < 4; ++z) o[n][b + z] *= alpha[n];
                }
                asm volatile("");
            }
        uint4 pt[NC][NT];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const float m_use = fmaxf(m_ref[n], -1e30f);  // nothing seen yet: finite exponents, weights 0
            float p[2][4];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const float off = FOLDED ? ev[y] - m_use : -m_use;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float s = x[n][y][r];
                    p[y][r] = __builtin_amdgcn_exp2f(SCALED ? fmaf(s, ks[y], off) : s + off);
                    if (F32) l_run[n][0] += p[y][r];
                    if (INT8 && F32) p[y][r] *= vup[y];
                }
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if (F32) {
                    float t[2][4];
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int r = 0; r < 4; ++r) t[y][r] = rest3(p[y][r], i);
                    pt[n][i] = make_uint4(uppers(t[0][0], t[0][1]), uppers(t[0][2], t[0][3]), uppers(t[1][0], t[1][1]), uppers(t[1][2], t[1][3]));
                } else {
                    pt[n][i] = make_uint4(pack_bf16_rne(p[0][0], p[0][1]), pack_bf16_rne(p[0][2], p[0][3]), pack_bf16_rne(p[1][0], p[1][1]),
                                          pack_bf16_rne(p[1][2], p[1][3]));
                    uint4 ones = make_uint4(one[0], one[0], one[1], one[1]);
                    l_run[n] = mfma32(*reinterpret_cast<bf16x8*>(&ones), *reinterpret_cast<bf16x8*>(&pt[n][i]), l_run[n]);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            uint4 vw = s_v[buf][b][lane];
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int i = 0; i < NT; ++i) o[n][b] = mfma32(*reinterpret_cast<bf16x8*>(&vw), *reinterpret_cast<bf16x8*>(&pt[n][i]), o[n][b]);
        }
    };

    if (st0 < st1) {
        fetch();
        load(st0, 0);
        lds_barrier();  // s_marked is 0
        put(0);
        for (int st = st0; st < st1; ++st) {
            const int buf = (st - st0) & 1;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                pages[u] = next_pages[u];
                cur_exps[u] = exps[u];
            }
            if (FMT == kFmtBf16) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the keys that went to LDS by themselves
            lds_barrier();                                                        // the stage is whole, and its other buffer is no longer read
            load(min(st + 1, st1 - 1), buf ^ 1);  // without a branch, so that nobody waits for it before it is put
            compute(buf);
            if (st + 1 < st1) put(buf ^ 1);
        }
        // the last load has gone to LDS that nobody reads; it ends before the workgroup gives it up
        if (FMT == kFmtBf16) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            lds_barrier();
            if (s_marked) mark_not_finite<D, NC, 1>(a, span, tile_seen, btrow, c, st0 * 2, min(st1 * 2, span.n), col_lo, col_last, o);
        }
    }
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        float l = l_run[n][0];
        if (F32) {
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
        }
        const int ci = wc + n * 16 + col, tq = ci / a.G, h = ci - tq * a.G;
        if (ci >= live) continue;
        if (a.splits == 1) {
            const float by = 1.f / (l > 0.f || l != l ? l : 1.f);
#pragma unroll
            for (int b = 0; b < NB; ++b)
                store_row<D, F32>(a, (int64_t)m.r0 + m.t0 + tq, c * a.G + h, b * 16 + lg * 4, o[n][b] * by);
        } else {
            const int64_t at = (((int64_t)slot * n_kv + c) * a.splits + split) * kManyCols + ci;
            if (lg == 0) {
                a.many_ml[at * 2] = fmaxf(m_ref[n], -1e30f);
                a.many_ml[at * 2 + 1] = l;
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) *reinterpret_cast<floatx4*>(a.many_o + at * D + b * 16 + lg * 4) = o[n][b];
        }
    }
}

// joins the parts of a tile: a workgroup per (slot, KV head, 8 or 16 columns), a quarter of a wave or half of one to a column
template <int D, bool F32>
__global__ __launch_bounds__(256) void row_many_merge_kernel(RowAttnArgs a) {
    constexpr int LANES = D / 4, S = 256 / LANES, GROUPS = kManyCols / S;
    const int g = blockIdx.x % GROUPS, rest = blockIdx.x / GROUPS, c = rest % a.n_kv, slot = rest / a.n_kv;
    ManyTile m;
    if (!many_tile(a, slot, m)) return;
    const int ci = g * S + threadIdx.x / LANES, ln = threadIdx.x % LANES;
    if (ci >= a.G * m.tv) return;
    const int64_t at0 = ((int64_t)slot * a.n_kv + c) * a.splits * kManyCols + ci;
    float M = -1e30f, den = 0.f;
    floatx4 num = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAtOnce = 4;  // parts whose loads are on their way together
    for (int j0 = 0; j0 < a.splits; j0 += kAtOnce) {
        float2 ml[kAtOnce];
        floatx4 o[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t at = at0 + (int64_t)min(j0 + u, a.splits - 1) * kManyCols;
            ml[u] = *reinterpret_cast<const float2*>(a.many_ml + at * 2);
            o[u] = *reinterpret_cast<const floatx4*>(a.many_o + at * D + ln * 4);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (j0 + u < a.splits) {
                const float Mn = fmaxf(M, ml[u].x), f0 = __builtin_amdgcn_exp2f(M - Mn), f1 = __builtin_amdgcn_exp2f(ml[u].x - Mn);
                num = num * f0 + o[u] * f1;
                den = den * f0 + ml[u].y * f1;
                M = Mn;
            }
    }
    if (!(den > 0.f) && den == den) den = 1.f;
    const int tq = ci / a.G, h = ci - tq * a.G;
    store_row<D, F32>(a, (int64_t)m.r0 + m.t0 + tq, c * a.G + h, ln * 4, num * (1.f / den));
}

// ---- host ---------------------------------------------------------------------------------------------------------

// How a call is laid out, from what the host knows
struct RowShape {
    int G, tg, few_max, cw, few_wgs, passes_max, tt, slots, splits_max;
    int64_t rec_bytes, few_ml, few_o, many_ml, many_o;  // bytes
    int64_t bytes() const { return rec_bytes + few_ml + few_o + many_ml + many_o; }
};
// Parts of a tile's pages, for that many workgroups (tile and KV head): the pages are dealt out where the compute unit that gets most workgroups has many more
// than the mean (a part more costs about 2 %).
constexpr int kSplitBelow = 4 * kNumCU;  // workgroups from which they never are
static int splits_for(int64_t wgs) {
    if (wgs >= kSplitBelow) return 1;
    int most = 1;
    double best = 1e30;
    for (int k = 1; k <= 16; ++k) {
        const double per = (double)wgs / kNumCU * k, cost = std::ceil(per) / per * (1.0 + 0.02 * (k - 1));
        if (cost < best - 1e-9) best = cost, most = k;
    }
    return most;
}
// the parts that calls of up to so many workgroups keep: fewer workgroups may be dealt out further and keep more
static int64_t parts_upto(int64_t wgs) {
    static const std::array<int, kSplitBelow> most = [] {
        std::array<int, kSplitBelow> m;
        m[0] = 0;
        for (int w = 1; w < kSplitBelow; ++w) {
            const int k = splits_for(w);
            m[w] = std::max(m[w - 1], k > 1 ? w * k : 0);
        }
        return m;
    }();
    return most[std::min<int64_t>(wgs, kSplitBelow - 1)];
}
static int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }
// its sizes have room for every call whose batch, rows and max_new are no larger
static RowShape row_shape(int n_q, int n_kv, int d, int batch, int rows, int max_new, int passes) {
    RowShape s;
    max_new = std::min(max_new, rows);
    s.G = n_q / n_kv;
    s.tg = std::max(1, 16 / s.G);
    s.few_max = passes * s.tg;
    const int cols = s.G * std::min(s.tg, max_new);
    s.cw = cols <= 4 ? 4 : cols <= 8 ? 8 : 16;
    s.few_wgs = std::max(1, 2 * kNumCU / n_kv);  // of a KV head
    s.passes_max = (int)std::min((int64_t)rows, (int64_t)batch * ((std::min(max_new, s.few_max) + s.tg - 1) / s.tg));
    s.rec_bytes = up16(16 + 16 * (int64_t)s.passes_max);
    const int64_t parts = (4 * (int64_t)s.few_wgs + s.passes_max) * n_kv * s.cw;
    s.few_ml = up16(parts * 8);
    s.few_o = parts * d * 4;
    s.tt = s.slots = s.splits_max = 0;
    s.many_ml = s.many_o = 0;
    if (max_new > s.few_max) {
        s.tt = kManyCols / s.G;
        s.slots = (int)((int64_t)rows / s.tt + std::min((int64_t)batch, (int64_t)rows / (s.few_max + 1)));  // tiles, at most: as many slots
        s.splits_max = splits_for((int64_t)s.slots * n_kv);
        const int64_t columns = parts_upto((int64_t)s.slots * n_kv) * kManyCols;
        s.many_ml = columns * 8;
        s.many_o = columns * d * 4;
    }
    return s;
}

// Up to how many passes a request is row_few_kernel's.  us by passes / by tiles: 32 requests of 4000 tokens, 4 heads to a KV head of 128: fp32 over int8 at
// 2 passes 104 / 165, 4 141 / 172, 8 239 / 312; fp32 over bf16 188 / 192, 222 / 194, 342 / 346; bf16 over int8 103 / 107, 137 / 115, 224 / 198; bf16 over bf16
// at 2 183 / 141.  8 heads to a KV head of 64: bf16 over bf16 33 / 45, 55 / 30; bf16 over e4m3 26 / 45, 37 / 32.  One request of 8000 tokens, whose tiles leave
// most compute units idle: 128 dims, 8 passes, fp32 over int8 38 / 48, bf16 over int8 36 / 36; over bf16 fp32 at 4 43 / 47, at 8 58 / 50, bf16 at 2 23 / 32, at
// 4 35 / 33; 64 dims at 8 passes 17 to 20 / 25 to 33.
constexpr int kMostPasses = 8;
static int few_passes(const chiron_attn_rows* in, int n_kv, int d, int format) {
    const bool wide = format == kFmtBf16 && d == 128, f32 = in->dtype == CHIRON_F32;
    if ((int64_t)in->batch * n_kv <= kNumCU / 8) return !wide ? kMostPasses : f32 ? 4 : 2;
    return f32 && format != kFmtBf16 ? kMostPasses : wide && !f32 ? 1 : 2;
}

template <int D, int FMT, bool F32, bool MULTI>
static void launch_few(const RowAttnArgs& a, const RowShape& s, hipStream_t st) {
    constexpr bool TERMS = F32 || FMT == kFmtInt8;
    const dim3 grid((unsigned)(s.few_wgs * a.n_kv));
    if (!TERMS || s.cw == 16) launch(row_few_kernel<D, FMT, F32, 16, MULTI>, grid, dim3(256), st, a);
    else if (s.cw == 8) launch(row_few_kernel<D, FMT, F32, TERMS ? 8 : 16, MULTI>, grid, dim3(256), st, a);
    else launch(row_few_kernel<D, FMT, F32, TERMS ? 4 : 16, MULTI>, grid, dim3(256), st, a);
    launch(row_few_merge_kernel<D, F32>, dim3((unsigned)((int64_t)s.passes_max * a.n_kv * a.pcols)), dim3(256), st, a);
}
template <int D, int FMT, bool F32>
static void launch_rows(const RowAttnArgs& a, const RowShape& s, hipStream_t st) {
    if (s.slots) {
        launch(row_many_kernel<D, FMT, F32>, dim3((unsigned)((int64_t)s.slots * a.splits * a.n_kv)), dim3(256), st, a);
        if (a.splits > 1) launch(row_many_merge_kernel<D, F32>, dim3((unsigned)((int64_t)s.slots * a.n_kv * (kManyCols * D / 1024))), dim3(256), st, a);
    }
    if (a.few_max == 0) return;
    if (a.max_new > 1) launch_few<D, FMT, F32, true>(a, s, st);
    else launch_few<D, FMT, F32, false>(a, s, st);
}
template <int FMT>
static void launch_format(const RowAttnArgs& a, const RowShape& s, int d, bool f32, hipStream_t st) {
    if (d == 128 && f32) launch_rows<128, FMT, true>(a, s, st);
    else if (d == 128) launch_rows<128, FMT, false>(a, s, st);
    else if (f32) launch_rows<64, FMT, true>(a, s, st);
    else launch_rows<64, FMT, false>(a, s, st);
}

static int32_t row_attention(const chiron_attn_rows* in, int n_kv, int d, int num_blocks, int format, const void* tiles, const int8_t* exps,
                             void* workspace, hipStream_t st) {
    if (in->batch < 0 || in->rows < 0 || in->max_new < 0) return fail(CHIRON_ERR_INVALID_ARG, "row attention: a size is negative");
    if (in->window < 0 || in->n_sinks < 0) return fail(CHIRON_ERR_INVALID_ARG, "row attention: window %d, n_sinks %d", in->window, in->n_sinks);
    if (in->dtype != CHIRON_F32 && in->dtype != CHIRON_BF16) return fail(CHIRON_ERR_INVALID_ARG, "row attention: dtype %d is neither CHIRON_F32 nor CHIRON_BF16", in->dtype);
    if (in->n_q_heads < 1 || in->n_q_heads % n_kv != 0 || in->n_q_heads / n_kv > 16)
        return fail(CHIRON_ERR_SHAPE, "row attention: %d query heads over %d KV heads: a multiple of them, at most 16 times as many", in->n_q_heads, n_kv);
    if (in->rows == 0 || in->max_new == 0) return CHIRON_OK;
    if (in->batch == 0) return fail(CHIRON_ERR_INVALID_ARG, "row attention: %d rows of no request", in->rows);
    if (!in->q || !in->out || !in->block_table || !in->row_starts || !in->seq_lens)
        return fail(CHIRON_ERR_INVALID_ARG, "row attention: a pointer argument is null");
    if (in->max_blocks_per_seq < 1 || in->max_blocks_per_seq > 1 << 26)
        return fail(CHIRON_ERR_INVALID_ARG, "row attention: max_blocks_per_seq %d is not in 1 .. 2^26", in->max_blocks_per_seq);
    const int size = in->dtype == CHIRON_F32 ? 4 : 2;
    if (in->q_stride < (int64_t)in->n_q_heads * d || in->q_stride * size % 16 != 0)
        return fail(CHIRON_ERR_INVALID_ARG, "row attention: q_stride %lld is smaller than a row or no multiple of 16 bytes", (long long)in->q_stride);
    if (((uintptr_t)in->q | (uintptr_t)in->out | (uintptr_t)workspace) & 15) return fail(CHIRON_ERR_INVALID_ARG, "row attention: q, out and the workspace must be 16-byte aligned");
    if (!workspace) return fail(CHIRON_ERR_INVALID_ARG, "row attention: the workspace is null");
    const uint64_t q0 = (uint64_t)(uintptr_t)in->q, o0 = (uint64_t)(uintptr_t)in->out, row = (uint64_t)in->n_q_heads * d * size;
    if (q0 < o0 + (uint64_t)in->rows * row && o0 < q0 + (uint64_t)(in->rows - 1) * (uint64_t)in->q_stride * size + row)
        return fail(CHIRON_ERR_INVALID_ARG, "row attention: out overlaps q, which other workgroups still read");
    const RowShape s = row_shape(in->n_q_heads, n_kv, d, in->batch, in->rows, in->max_new, few_passes(in, n_kv, d, format));
    if ((int64_t)s.passes_max * in->max_blocks_per_seq >= (int64_t)1 << 31)
        return fail(CHIRON_ERR_SHAPE, "row attention: %d requests of up to %d pages are too many for one call", in->batch, in->max_blocks_per_seq);
    RowAttnArgs a = {};
    a.tiles = (const uint8_t*)tiles; a.exps = exps;
    a.q = in->q; a.out = in->out; a.q_stride = in->q_stride;
    a.bt = in->block_table; a.row_starts = in->row_starts; a.seq_lens = in->seq_lens;
    a.window = in->window ? in->window : (int64_t)1 << 40;
    a.num_blocks = num_blocks; a.n_kv = n_kv; a.G = s.G; a.max_blocks = in->max_blocks_per_seq; a.batch = in->batch; a.rows = in->rows;
    a.max_new = in->max_new; a.n_sinks = in->n_sinks;
    a.scale_log2e = (float)(1.4426950408889634 / std::sqrt((double)d));
    a.few_max = s.few_max; a.tg = s.tg; a.pcols = s.cw; a.passes_max = s.passes_max; a.tt = s.tt;
    // one request that may bring many rows goes by tiles even if it brings few: the two launches for few rows cost 9 us; one that then brings a single
    // row pays a tile's padding
    if (s.slots && in->batch == 1) a.few_max = 0;
    a.splits = 1;
    if (s.splits_max > 1) {  // a part has 256 tokens at least, if the window or the table lets a tile see as many
        int64_t pages = in->max_blocks_per_seq;
        if (in->window) pages = std::min(pages, ((int64_t)in->window + s.tt) / kBlockSize + in->n_sinks / kBlockSize + 3);
        a.splits = (int)std::min<int64_t>(s.splits_max, std::max<int64_t>(1, pages / 16));
    }
    if ((int64_t)s.slots * std::max(a.splits, 16) * n_kv > 0x7fffffff || (int64_t)s.passes_max * n_kv * s.cw > 0x7fffffff)
        return fail(CHIRON_ERR_SHAPE, "row attention: %d rows are too many for one call", in->rows);
    uint8_t* ws = (uint8_t*)workspace;
    a.head = (int32_t*)ws;
    a.part_ml = (float*)(ws + s.rec_bytes);
    a.part_o = (float*)(ws + s.rec_bytes + s.few_ml);
    a.many_ml = (float*)(ws + s.rec_bytes + s.few_ml + s.few_o);
    a.many_o = (float*)(ws + s.rec_bytes + s.few_ml + s.few_o + s.many_ml);
    const bool f32 = in->dtype == CHIRON_F32;
    if (format == kFmtBf16) launch_format<kFmtBf16>(a, s, d, f32, st);
    else if (format == kFmtInt8) launch_format<kFmtInt8>(a, s, d, f32, st);
    else launch_format<kFmtE4m3>(a, s, d, f32, st);
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

}  // namespace chiron

using namespace chiron;

extern "C" {

int64_t chiron_row_attention_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t batch, int32_t rows, int32_t max_new) {
    if (n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads != 0 || n_q_heads / n_kv_heads > 16 || (head_dim != 64 && head_dim != 128)) return 0;
    if (batch < 1 || rows < 1 || max_new < 1) return 0;
    int64_t most = 0;  // whatever the pool and the type are, and for smaller calls too
    for (int passes = 1; passes <= kMostPasses; passes *= 2) most = std::max(most, row_shape(n_q_heads, n_kv_heads, head_dim, batch, rows, max_new, passes).bytes());
    return most;
}

int32_t chiron_op_row_attention(const chiron_kvpool* p, int32_t layer, const chiron_attn_rows* in, void* workspace, void* stream) {
    if (!p || !in) return fail(CHIRON_ERR_INVALID_ARG, "pool or rows is null");
    if (layer < 0 || layer >= p->d.n_layers) return fail(CHIRON_ERR_INVALID_ARG, "layer %d out of range", layer);
    return row_attention(in, p->d.n_kv, p->d.d, p->d.num_blocks, kFmtBf16, p->d.base + (int64_t)layer * p->d.layer_stride, nullptr, workspace, (hipStream_t)stream);
}

int32_t chiron_op_row_attention8(const chiron_kvpool8* p, int32_t layer, const chiron_attn_rows* in, void* workspace, void* stream) {
    if (!p || !in) return fail(CHIRON_ERR_INVALID_ARG, "pool or rows is null");
    if (layer < 0 || layer >= p->d.n_layers) return fail(CHIRON_ERR_INVALID_ARG, "layer %d out of range", layer);
    const uint8_t* base = p->d.base + (int64_t)layer * p->d.layer_stride;
    return row_attention(in, p->d.n_kv, p->d.d, p->d.num_blocks, p->d.format, base, (const int8_t*)base + p->d.exps_at, workspace, (hipStream_t)stream);
}

}  // extern "C"
