// Verification of drafted tokens: acceptance against the target's probabilities and the token that replaces the first rejected one.
// gfx950, wave64.
//
// Two launches.  (1) Every logit row's maximum, its index, and sum of exponentials, in pieces over the vocabulary: the only pass
// over all rows, bounded by reading them.  (2) A workgroup per request and piece joins the pieces of its request's rows, decides how
// many drafts are taken (every workgroup of a request comes to the same answer from the same numbers), and races what is left of the
// vocabulary in its piece; the two or three rows it needs again come from the caches.  The pieces' winners meet in an
// atomic maximum, and the workgroup of a request that comes last writes the token.
// 64 requests of 4 drafts over 128256 tokens: 46 us (6.4 TB/s) and 23; one request: 5.6 and 8.6, a chain of loads that wait for one
// another.  (A third launch for the winners, and the decision in one thread's loop, took 5 us more, with one request and with 23.)
// The race argmax r(x)/noise(x) instead of a running sum over the vocabulary: it is one pass in any order, and which token wins does
// not depend on the order of any sum.
#include <new>

#include "draft_ops.h"

namespace chiron {

constexpr float kTopF32 = 3.4028234663852886e38f;
constexpr int kMaxDrafts = 127;
constexpr int kVerifyThreads = 256;
constexpr int kVerifyPiece = 4096;  // logits of a row per workgroup

struct RowStat {
    float m, z;  // maximum; sum of exp((x - m) / T)
    int best;    // lowest index of the maximum, -1: nothing above -inf
    int pad;
};
// The best r/noise of a request: bit 63 where the draft was taken off p and something is left, which beats all of p; the value's bits (it
// is not negative) over 2^32 - 1 - token, so that of equal ones the lower token is more; 0: none.  The maximum does not depend on the
// order in which the pieces come.
struct Winner {
    unsigned long long key;
    uint32_t arrived, pad;  // pieces
};
__device__ __forceinline__ unsigned long long race_key(bool rest, float v, int token) {
    return (unsigned long long)rest << 63 | (unsigned long long)__float_as_uint(v) << 32 | (0xffffffffu - (uint32_t)token);
}

template <int Ctrl>
__device__ __forceinline__ unsigned long long moved(unsigned long long key) {
    return (unsigned long long)(uint32_t)row_move<Ctrl>((int)(key >> 32)) << 32 | (uint32_t)row_move<Ctrl>((int)key);
}
struct VerifyArgs {
    chiron_draft_batch in;
    int batch, max_draft, vocab, pieces;
    RowStat* stats;  // [batch][2*max_draft+1][pieces]: target rows, then draft rows
    Winner* winners; // [batch], made ready by the first launch
    int32_t *out_tokens, *accepted;
    float* prob;
};

// exp(d / T) with c = log2(e) / T by one product and the machine's exponential: off by up to |d / T| 2^-22 + 2^-23 of itself, as c has three
// roundings and the product one.  In a sum that is much only where the term is small.
__device__ __forceinline__ float weight(float d, float c) { return __builtin_amdgcn_exp2f(d * c); }
__device__ __forceinline__ float log2e_over(float inv_t) { return fminf(inv_t * 1.44269504088896341f, kTopF32); }
__device__ __forceinline__ float logit_of(float x) { return x != x ? -INFINITY : fminf(x, kTopF32); }
// 1 / T of a request; 0: greedy.  A temperature above 0 never comes out as that: 1 / inf is taken as the least number above 0, which
// leaves logits that are no infinity alike and those of -inf at -inf.
constexpr float kLeastF32 = 1.401298464324817e-45f;
__device__ __forceinline__ float inv_temperature(const VerifyArgs& a, int i) {
    if (!a.in.temperature) return 1.f;
    const float t = a.in.temperature[i];
    return t > 0.f ? fmaxf(fminf(1.f / t, kTopF32), kLeastF32) : 0.f;
}
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int i) {
    return a.in.draft_lens ? min(max(a.in.draft_lens[i], 0), a.max_draft) : a.max_draft;
}
// joins two statistics of one row; of equal maxima the lower index
__device__ __forceinline__ void join(float& m, float& z, int& best, float m2, float z2, int best2, float c) {
    if (m2 == -INFINITY) return;
    if (m == -INFINITY) {
        m = m2; z = z2; best = best2;
        return;
    }
    if (m2 > m) {
        z = z * weight(m - m2, c) + z2;
        m = m2;
        best = best2;
    } else {
        z += z2 * weight(m2 - m, c);
        if (m2 == m) best = min(best, best2);
    }
}
// joins over 16 neighbouring lanes, or all 64: every step with a lane that has joined others
template <int Ctrl>
__device__ __forceinline__ void join_moved(float& m, float& z, int& best, float c) {
    const float m2 = row_move<Ctrl>(m), z2 = row_move<Ctrl>(z);
    join(m, z, best, m2, z2, row_move<Ctrl>(best), c);
}
template <int LANES>
__device__ __forceinline__ void join_lanes(float& m, float& z, int& best, float c) {
#pragma unroll
    for (int o = LANES / 2; o >= 16; o >>= 1) {
        const float m2 = __shfl_xor(m, o), z2 = __shfl_xor(z, o);
        const int b2 = __shfl_xor(best, o);
        join(m, z, best, m2, z2, b2, c);
    }
    join_moved<kRor8>(m, z, best, c);
    join_moved<kRor4>(m, z, best, c);
    join_moved<kRor2>(m, z, best, c);
    join_moved<kRor1>(m, z, best, c);
}

// Rows of any length begin at any multiple of 4 bytes: a piece is 1024 vectors of 16 bytes counted from the 16-byte boundary at or
// before the row's start, and only vectors that lie wholly within the row are loaded as such.
__global__ __launch_bounds__(kVerifyThreads) void verify_stats_kernel(VerifyArgs a) {
    __shared__ float s_m[4], s_z[4];
    __shared__ int s_b[4];
    const int rows = 2 * a.max_draft + 1;
    const int i = blockIdx.y / rows, r = blockIdx.y % rows, piece = blockIdx.x;
    const int n = drafts_of(a, i);
    const float inv_t = inv_temperature(a, i), c = log2e_over(inv_t);
    const bool draft = r > a.max_draft;
    const int t = draft ? r - a.max_draft - 1 : r;
    if (draft ? (t >= n || !a.in.draft_logits || inv_t == 0.f) : t > n) return;  // nobody asks for this row
    if (r == 0 && piece == 0 && threadIdx.x == 0) a.winners[i] = Winner{0, 0, 0};
    const float* row = draft ? a.in.draft_logits + ((int64_t)i * a.max_draft + t) * a.in.draft_stride
                             : a.in.logits + ((int64_t)i * (a.max_draft + 1) + t) * a.in.logits_stride;
    const int shift = (int)((uintptr_t)row >> 2 & 3);
    constexpr int VPT = kVerifyPiece / kVerifyThreads / 4;
    float4 v[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int x = (piece * (kVerifyPiece / 4) + j * kVerifyThreads + threadIdx.x) * 4 - shift;
        if (x >= 0 && x + 4 <= a.vocab) v[j] = *reinterpret_cast<const float4*>(row + x);
        else {
            float* p = &v[j].x;
#pragma unroll
            for (int k = 0; k < 4; ++k) p[k] = x + k >= 0 && x + k < a.vocab ? row[x + k] : -INFINITY;
        }
    }
    float m = -INFINITY, z = 0.f;
    int best = -1;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        float* p = &v[j].x;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            p[k] = logit_of(p[k]);
            if (p[k] > m) {
                m = p[k];
                best = (piece * (kVerifyPiece / 4) + j * kVerifyThreads + threadIdx.x) * 4 - shift + k;
            }
        }
    }
    if (m > -INFINITY)
#pragma unroll
        for (int j = 0; j < VPT; ++j) z += (weight(v[j].x - m, c) + weight(v[j].y - m, c)) + (weight(v[j].z - m, c) + weight(v[j].w - m, c));
    join_lanes<64>(m, z, best, c);
    if ((threadIdx.x & 63) == 0) {
        s_m[threadIdx.x >> 6] = m;
        s_z[threadIdx.x >> 6] = z;
        s_b[threadIdx.x >> 6] = best;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kVerifyThreads / 64; ++w) join(m, z, best, s_m[w], s_z[w], s_b[w], c);
        a.stats[(int64_t)blockIdx.y * a.pieces + piece] = RowStat{m, z, best, 0};
    }
}

// p(x) of a row
__device__ __forceinline__ float share(float x, float m, float z, float inv_t) {
    return z > 0.f ? expf((logit_of(x) - m) * inv_t) / z : 0.f;
}

__global__ __launch_bounds__(kVerifyThreads) void verify_race_kernel(VerifyArgs a) {
    __shared__ RowStat s_row[2 * kMaxDrafts + 1];
    __shared__ int s_tok[kMaxDrafts], s_first[2];
    __shared__ unsigned long long s_key[kVerifyThreads / 64];
    const int i = blockIdx.y, piece = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t0 = threadIdx.x;
    const int rows = 2 * a.max_draft + 1;
    const float* target = a.in.logits + (int64_t)i * (a.max_draft + 1) * a.in.logits_stride;
    const float* draft = a.in.draft_logits ? a.in.draft_logits + (int64_t)i * a.max_draft * a.in.draft_stride : nullptr;
    const int32_t* tok = a.in.tokens + (int64_t)i * a.max_draft;
    // A chain of loads, each a microsecond, is what this kernel takes with few requests: what does not wait for the rows' sums and the
    // decision is on its way first.
    const int x0 = piece * kVerifyPiece + t0;
    constexpr int VPT = kVerifyPiece / kVerifyThreads;
    float noise[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) noise[j] = x0 + j * kVerifyThreads < a.vocab ? a.in.noise[(int64_t)i * a.vocab + x0 + j * kVerifyThreads] : 1.f;
    int my_tok = -1;
    float my_target = 0.f, my_draft = 0.f, my_uniform = 0.f;
    if (t0 < a.max_draft) {
        my_tok = s_tok[t0] = tok[t0];
        my_uniform = a.in.uniforms[(int64_t)i * a.max_draft + t0];
        if (my_tok >= 0 && my_tok < a.vocab) {
            my_target = target[t0 * a.in.logits_stride + my_tok];
            if (draft) my_draft = draft[t0 * a.in.draft_stride + my_tok];
        } else my_tok = -1;
    }
    const int n = drafts_of(a, i);
    const float inv_t = inv_temperature(a, i), c = log2e_over(inv_t);
    const bool greedy = inv_t == 0.f, with_draft = draft && !greedy;
    const int need = n + 1 + (with_draft ? n : 0);
    // 16 lanes join a row's pieces
    for (int w = t0 / 16; w - t0 / 16 < need; w += kVerifyThreads / 16) {
        const int r = w <= n ? w : a.max_draft + w - n;  // target rows 0..n, then the draft's 0..n-1
        float m = -INFINITY, z = 0.f;
        int best = -1;
        if (w < need) {
            const RowStat* st = a.stats + ((int64_t)i * rows + r) * a.pieces;
            for (int p = t0 % 16; p < a.pieces; p += 16) {
                const RowStat s = st[p];
                join(m, z, best, s.m, s.z, s.best, c);
            }
        }
        join_lanes<16>(m, z, best, c);
        if (w < need && t0 % 16 == 0) s_row[w] = RowStat{m, z, best, 0};
    }
    __syncthreads();
    static_assert(kMaxDrafts <= 128, "a lane of the first two waves for each draft");
    float pr = 0.f;
    if (t0 < n && my_tok >= 0) {
        const RowStat p = s_row[t0];
        if (greedy) pr = my_tok == p.best ? 1.f : 0.f;
        else {
            const float px = share(my_target, p.m, p.z, inv_t);
            if (with_draft) {
                const RowStat q = s_row[n + 1 + t0];
                const float qx = share(my_draft, q.m, q.z, inv_t);
                pr = qx > 0.f ? fminf(1.f, px / qx) : px > 0.f ? 1.f : 0.f;
            } else pr = px;
        }
    }
    if (wave < 2) {
        const unsigned long long refused = __ballot(t0 < n && !(my_uniform < pr));
        if (lane == 0) s_first[wave] = refused ? wave * 64 + __builtin_ctzll(refused) : kMaxDrafts;
    }
    __syncthreads();
    const int took = min(n, min(s_first[0], s_first[1]));
    if (piece == 0 && t0 <= a.max_draft) {
        if (a.prob && t0 < a.max_draft) a.prob[(int64_t)i * a.max_draft + t0] = pr;
        if (t0 != took) a.out_tokens[(int64_t)i * (a.max_draft + 1) + t0] = t0 < took ? s_tok[t0] : -1;
        if (t0 == 0) a.accepted[i] = took;
    }
    const RowStat p = s_row[took];
    float best_rest = -1.f, best_all = -1.f;
    int rest_at = -1, all_at = -1;
    if (greedy) {
        best_all = 1.f;
        all_at = p.best;
    } else if (p.z > 0.f) {
        const bool rejected = took < n;
        const float* prow = target + took * a.in.logits_stride;
        const float* qrow = rejected && with_draft ? draft + took * a.in.draft_stride : nullptr;
        const RowStat q = qrow ? s_row[n + 1 + took] : RowStat{0.f, 0.f, -1, 0};
        const int without = rejected && !with_draft ? s_tok[took] : -1;
        float pv[VPT], qv[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) pv[j] = x0 + j * kVerifyThreads < a.vocab ? prow[x0 + j * kVerifyThreads] : -INFINITY;
        if (qrow)
#pragma unroll
            for (int j = 0; j < VPT; ++j) qv[j] = x0 + j * kVerifyThreads < a.vocab ? qrow[x0 + j * kVerifyThreads] : -INFINITY;
        // Exponentials and reciprocals of the machine's own precision: r / noise is off by up to |d / T| 2^-22 + 2^-21 of itself, 2^-16 for a
        // token with e^-50 of the largest share.  Only a race as close as that can go to the other token.
        const float rp = 1.f / p.z, rq = q.z > 0.f ? 1.f / q.z : 0.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int x = x0 + j * kVerifyThreads;
            const float inv = __builtin_amdgcn_rcpf(noise[j]);
            const float ps = weight(logit_of(pv[j]) - p.m, c) * rp;
            float rest = ps;
            if (qrow) rest = fmaxf(ps - (rq > 0.f ? weight(logit_of(qv[j]) - q.m, c) * rq : 0.f), 0.f);
            else if (x == without) rest = 0.f;
            const float all = ps * inv, some = rest * inv;
            if (ps > 0.f && all > best_all) {
                best_all = all;
                all_at = x;
            }
            if (rest > 0.f && some > best_rest) {
                best_rest = some;
                rest_at = x;
            }
        }
    }
    unsigned long long key = rest_at >= 0 ? race_key(true, best_rest, rest_at) : all_at >= 0 ? race_key(false, best_all, all_at) : 0;
    key = max(key, (unsigned long long)__shfl_xor(key, 32));
    key = max(key, (unsigned long long)__shfl_xor(key, 16));
    key = max(key, moved<kRor8>(key));
    key = max(key, moved<kRor4>(key));
    key = max(key, moved<kRor2>(key));
    key = max(key, moved<kRor1>(key));
    if (lane == 0) s_key[wave] = key;
    __syncthreads();
    if (t0 == 0) {
        for (int w = 1; w < kVerifyThreads / 64; ++w) key = max(key, s_key[w]);
        // No release or acquire, which write back and empty the whole L2 and make 23 us of 64 requests' race 75: nothing but these two
        // words passes between the workgroups, and the maximum has come back, so it is done, before the count goes out.
        Winner* win = a.winners + i;
        uint32_t one = 1;
        const unsigned long long was = __hip_atomic_fetch_max(&win->key, key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("" : "+v"(one) : "v"(was) : "memory");
        if (__hip_atomic_fetch_add(&win->arrived, one, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 != (uint32_t)a.pieces) return;
        key = __hip_atomic_fetch_max(&win->key, key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        a.out_tokens[(int64_t)i * (a.max_draft + 1) + took] = key ? (int)(0xffffffffu - (uint32_t)key) : -1;
    }
}

static int verify_pieces(int vocab) { return (int)(((int64_t)vocab + 3 + kVerifyPiece - 1) / kVerifyPiece); }  // up to 3 values before an aligned start

}  // namespace chiron

using namespace chiron;

extern "C" {

int64_t chiron_verify_workspace_bytes(int32_t batch, int32_t max_draft, int32_t vocab) {
    if (batch < 0 || max_draft < 0 || max_draft > kMaxDrafts || vocab < 1) return 0;
    return (int64_t)batch * (verify_pieces(vocab) * (2 * max_draft + 1) * (int64_t)sizeof(RowStat) + (int64_t)sizeof(Winner));
}

int32_t chiron_op_verify_drafts(const chiron_draft_batch* in, int32_t batch, int32_t max_draft, int32_t vocab, int32_t* out_tokens,
                                int32_t* accepted, float* prob, void* workspace, void* stream) {
    if (!in) return fail(CHIRON_ERR_INVALID_ARG, "verify: the batch is null");
    if (batch < 0 || max_draft < 0 || vocab < 1) return fail(CHIRON_ERR_INVALID_ARG, "verify: bad sizes");
    if (max_draft > kMaxDrafts) return fail(CHIRON_ERR_SHAPE, "verify: %d drafted tokens, at most %d", max_draft, kMaxDrafts);
    if (batch == 0) return CHIRON_OK;
    if (!in->logits || !in->noise || !out_tokens || !accepted || !workspace || (max_draft > 0 && (!in->tokens || !in->uniforms)))
        return fail(CHIRON_ERR_INVALID_ARG, "verify: a pointer is null");
    if (in->logits_stride < vocab || (in->draft_logits && in->draft_stride < vocab))
        return fail(CHIRON_ERR_INVALID_ARG, "verify: a row stride is smaller than the vocabulary");
    if ((uintptr_t)workspace & 15) return fail(CHIRON_ERR_INVALID_ARG, "verify: the workspace must be 16-byte aligned");
    const int pieces = verify_pieces(vocab);
    const int64_t rows = (int64_t)batch * (2 * max_draft + 1);
    if (rows > 65535) return fail(CHIRON_ERR_BATCH_TOO_LARGE, "verify: %d requests of %d drafts are too many for one call", batch, max_draft);
    VerifyArgs a;
    a.in = *in;
    a.batch = batch; a.max_draft = max_draft; a.vocab = vocab; a.pieces = pieces;
    a.stats = (RowStat*)workspace;
    a.winners = (Winner*)((char*)workspace + rows * pieces * (int64_t)sizeof(RowStat));
    a.out_tokens = out_tokens; a.accepted = accepted; a.prob = prob;
    hipStream_t st = (hipStream_t)stream;
    launch(verify_stats_kernel, dim3(pieces, (unsigned)rows), dim3(kVerifyThreads), st, a);
    launch(verify_race_kernel, dim3(pieces, batch), dim3(kVerifyThreads), st, a);
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

}  // extern "C"
