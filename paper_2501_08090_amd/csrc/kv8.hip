// The cache in 8 bits: rotate-and-append with a power of two for each page and KV head, and the read-back.  gfx950, wave64.
//
// A wave owns one (page, KV head), as in the bf16 append, so that it knows the largest value of the page's new tokens, and writes the
// codes in pieces of 8 bytes (K) and 16 (V).  A page that held tokens before keeps the larger power of two; only if that has
// grown are its old codes read, divided and rounded again.  Division by a power of two and the rounding are exact operations, so what is
// stored follows from the rotated values alone.
//
// Bound by memory where there are many rows: 16384 fp32 rows of 32 + 2 x 8 heads of 128 120 to 124 us, 700 MB at 5.7 TB/s, most of them the queries'; 5003 bf16 rows 28 to
// 33 us; 64 single tokens 7.7 us, a chain of loads (row starts, table entry, page, all at once from there on).  The read-back reads V's four tokens of a
// word for one, 4 us for 64 tokens, 27 for 16384.
#include <new>

#include "append_rows.h"
#include "cache8.h"

namespace chiron {

struct Append8Args : NewRowArgs {
    Pool8Desc pool;
};

// an old word of four codes with the power of two grown by 1 / down
template <int FMT>
__device__ __forceinline__ uint32_t coarser(uint32_t w, float down) {
    const floatx4 f = decode8<FMT>(w) * down;
    return encode8<FMT>(f[0], f[1], f[2], f[3]);
}

// the largest of a wave's values, none below 0
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, row_move<kRor8>(v));
    v = fmaxf(v, row_move<kRor4>(v));
    v = fmaxf(v, row_move<kRor2>(v));
    v = fmaxf(v, row_move<kRor1>(v));
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// workgroups 0 .. page_wgs-1: four (page slot, KV head) each; the others: queries
template <int D, int FMT, bool F32, bool VEC>
__global__ __launch_bounds__(256) void append8_rope_kernel(Append8Args a) {
    constexpr int H = D / 64;  // pieces of 8 dims per lane and half of a head; V words of 16 bytes per lane
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)blockIdx.x >= a.page_wgs) {
        if (a.stream) rotate_queries<D, F32, VEC, true>(a);
        else rotate_queries<D, F32, VEC, false>(a);
        return;
    }
    const int n_kv = a.pool.n_kv;
    const int64_t task = (int64_t)blockIdx.x * 4 + wave;
    const int slot = (int)(task / n_kv), kvh = (int)(task % n_kv);
    NewPage np;
    if (!new_page(a, slot, a.pool.num_blocks, np)) return;
    const int r0 = np.r0, r1 = np.r1, t0 = np.t0, t1 = np.t1;
    uint8_t* tile = tile8(a.pool, a.layer, np.block, kvh);
    uint8_t* vtile = tile + 16 * D;
    int8_t* exps = exps8(a.pool, a.layer, np.block, kvh);

    // Everything that the page needs is on its way before the first of it is used: rows outside the request are replaced by its first or
    // last, so that no load hangs on a branch.  First what the page has: its powers of two, and the words of V that keep old bytes.
    const uint32_t had_exps = *reinterpret_cast<const uint16_t*>(exps);
    uint4 had[H];
    if (t0 > 0 || t1 < kBlockSize) {
#pragma unroll
        for (int b = 0; b < H; ++b) had[b] = *reinterpret_cast<const uint4*>(vtile + v8_off(4 * (lane >> 4), 64 * b + (lane & 15)));
    }
    // V: lane = (dim l of 16, four tokens 4u ..); word b holds the dims 64b + 16j + l, j = 0 .. 3, of these tokens
    const int l = lane & 15, u = lane >> 4;
    float vx[H][4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const void* src = (const char*)a.v + min(max(np.row0 + 4 * u + i, (int64_t)r0), (int64_t)r1 - 1) * a.v_stride;
#pragma unroll
        for (int b = 0; b < H; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) vx[b][j][i] = load1<F32>(src, kvh * D + 64 * b + 16 * j + l);
    }
    // K: lane = (token t, group g): the pieces of 8 dims g, g + 4, ... of the lower half of the head, and their rotary partners
    const int t = lane & 15, g = lane >> 4;
    const int64_t r = min(max(np.row0 + t, (int64_t)r0), (int64_t)r1 - 1);
    float kx[H][8], ky[H][8];
    {
        float kc[H][8], ks[H][8];
#pragma unroll
        for (int p = 0; p < H; ++p) {
            const int e = (g + 4 * p) * 8;
            const void* src = (const char*)a.k + r * a.k_stride;
            load8<F32, VEC>(src, kvh * D + e, kx[p]);
            load8<F32, VEC>(src, kvh * D + e + D / 2, ky[p]);
            load8<true, true>(a.cos_t + r * (D / 2), e, kc[p]);
            load8<true, true>(a.sin_t + r * (D / 2), e, ks[p]);
        }
        const bool is_new = t >= t0 && t < t1;
#pragma unroll
        for (int p = 0; p < H; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const Turned w = turn(kx[p][i], ky[p][i], kc[p][i], ks[p][i]);
                kx[p][i] = is_new ? bounded8(w.a) : 0.f;
                ky[p][i] = is_new ? bounded8(w.b) : 0.f;
            }
    }
    const int ek_old = t0 > 0 ? (int8_t)(had_exps & 0xff) : kMinExp8, ev_old = t0 > 0 ? (int8_t)(had_exps >> 8) : kMinExp8;

    float top = 0.f, vtop = 0.f;
#pragma unroll
    for (int p = 0; p < H; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(kx[p][i]), fabsf(ky[p][i])));
#pragma unroll
    for (int b = 0; b < H; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool is_new = 4 * u + i >= t0 && 4 * u + i < t1;
                vx[b][j][i] = is_new ? bounded8(vx[b][j][i]) : 0.f;
                vtop = fmaxf(vtop, fabsf(vx[b][j][i]));
            }
    top = wave_max(top);
    vtop = wave_max(vtop);
    const int ek = max(ek_old, power8<FMT>(top)), ev = max(ev_old, power8<FMT>(vtop));
    const float kup = two_to(-ek), vup = two_to(-ev);
    // (a step that grew by more than 2^126 leaves nothing of an old code)
    const float kdown = two_to(max(ek_old - ek, -126)), vdown = two_to(max(ev_old - ev, -126));

    if (t < t1) {
        const bool old = t < t0;
#pragma unroll
        for (int p = 0; p < 2 * H; ++p) {
            const int e = (g + 4 * (p % H)) * 8 + p / H * (D / 2);
            uint2* dst = reinterpret_cast<uint2*>(tile + k8_off(t, e));
            if (!old) {
                const float* x = p < H ? kx[p % H] : ky[p % H];
                *dst = make_uint2(encode8<FMT>(x[0] * kup, x[1] * kup, x[2] * kup, x[3] * kup),
                                  encode8<FMT>(x[4] * kup, x[5] * kup, x[6] * kup, x[7] * kup));
            } else if (ek > ek_old) {
                const uint2 w = *dst;
                *dst = make_uint2(coarser<FMT>(w.x, kdown), coarser<FMT>(w.y, kdown));
            }
        }
    }
    if (4 * u < t1 && (4 * u + 4 > t0 || ev > ev_old)) {
        // bytes of the word that are new, and that are old
        const int n0 = min(max(t0 - 4 * u, 0), 4), n1 = min(max(t1 - 4 * u, 0), 4);
        const uint32_t upto0 = n0 == 4 ? ~0u : (1u << (8 * n0)) - 1, upto1 = n1 == 4 ? ~0u : (1u << (8 * n1)) - 1;
        const uint32_t fresh = upto1 & ~upto0;
#pragma unroll
        for (int b = 0; b < H; ++b) {
            uint4* dst = reinterpret_cast<uint4*>(vtile + v8_off(4 * u, 64 * b + l));
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = encode8<FMT>(vx[b][j][0] * vup, vx[b][j][1] * vup, vx[b][j][2] * vup, vx[b][j][3] * vup);
            if (fresh != ~0u) {
                const uint32_t h[4] = {had[b].x, had[b].y, had[b].z, had[b].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t kept = ev > ev_old ? (coarser<FMT>(h[j], vdown) & upto0) | (h[j] & ~upto0) : h[j];
                    w[j] = (w[j] & fresh) | (kept & ~fresh);
                }
            }
            *dst = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    if (lane == 0) {
        exps[0] = (int8_t)ek;
        exps[1] = (int8_t)ev;
    }
}

// a thread per (token, KV head, 16 dims of K and as many of V)
template <int FMT>
__global__ __launch_bounds__(256) void gather8_kernel(Pool8Desc pool, int layer, const int32_t* __restrict__ bt, int max_blocks,
                                                      const int32_t* __restrict__ seq_idx, const int32_t* __restrict__ pos, int64_t n,
                                                      uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int pieces = pool.d / 16;
    const int64_t th = j / pieces, tok = th / pool.n_kv;
    if (tok >= n) return;
    const int p = (int)(j % pieces), kvh = (int)(th % pool.n_kv), at = pos[tok];
    int block = -1;
    if (at >= 0 && at / kBlockSize < max_blocks) block = bt[(size_t)seq_idx[tok] * max_blocks + at / kBlockSize];
    const bool there = block >= 0 && block < pool.num_blocks;
    const int t = at & 15;
    uint4 k = make_uint4(0, 0, 0, 0);
    uint32_t v[4] = {0, 0, 0, 0};  // the four dims 64b + 16j + l of l = l0 .. l0+3, j in the bytes
    const int b = p / 4, l0 = p % 4 * 4;
    float ks = 0.f, vs = 0.f;
    if (there) {
        const uint8_t* tile = tile8(pool, layer, block, kvh);
        const int8_t* e = exps8(pool, layer, block, kvh);
        ks = two_to(e[0]);
        vs = two_to(e[1]);
        k = *reinterpret_cast<const uint4*>(tile + k8_off(t, p * 16));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 w = *reinterpret_cast<const uint4*>(tile + 16 * pool.d + v8_off(t & ~3, 64 * b + l0 + i));
            const int down = (t & 3) * 8;
            v[i] = (w.x >> down & 0xff) | (w.y >> down & 0xff) << 8 | (w.z >> down & 0xff) << 16 | (w.w >> down) << 24;
        }
    }
    uint16_t *kd = k_out + th * pool.d + p * 16, *vd = v_out + th * pool.d + 64 * b + l0;
    const uint32_t kw[4] = {k.x, k.y, k.z, k.w};
    floatx4 vf[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const floatx4 f = decode8<FMT>(kw[i]) * ks;
        *reinterpret_cast<uint2*>(kd + 4 * i) = make_uint2(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]));
        vf[i] = decode8<FMT>(v[i]) * vs;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint2*>(vd + 16 * i) = make_uint2(pack_bf16_rne(vf[0][i], vf[1][i]), pack_bf16_rne(vf[2][i], vf[3][i]));
}

static Pool8Desc pool8_layout(const chiron_model* m, int32_t num_blocks) {
    Pool8Desc p;
    p.num_blocks = num_blocks;
    p.n_kv = m->cfg.n_kv_heads;
    p.d = m->cfg.head_dim;
    p.n_layers = m->cfg.n_layers;
    const int64_t tiles = (int64_t)num_blocks * p.n_kv;
    p.exps_at = tiles * 32 * p.d;
    p.layer_stride = (p.exps_at + tiles * 2 + 255) / 256 * 256;
    return p;
}

}  // namespace chiron

using namespace chiron;

extern "C" {

int64_t chiron_kv8_pool_bytes(const chiron_model* m, int32_t num_blocks) {
    if (!m || num_blocks < 1) return 0;
    const Pool8Desc p = pool8_layout(m, num_blocks);
    return p.layer_stride * p.n_layers;
}

int32_t chiron_kv8_pool_create(const chiron_model* m, void* dev_mem, uint64_t bytes, int32_t num_blocks, int32_t format, chiron_kvpool8** out) {
    if (!out) return fail(CHIRON_ERR_INVALID_ARG, "out is null");
    *out = nullptr;
    if (!m || !dev_mem) return fail(CHIRON_ERR_INVALID_ARG, "model or dev_mem is null");
    if (num_blocks < 1) return fail(CHIRON_ERR_INVALID_ARG, "num_blocks must be positive");
    if (format != CHIRON_INT8 && format != CHIRON_E4M3) return fail(CHIRON_ERR_INVALID_ARG, "format %d is neither CHIRON_INT8 nor CHIRON_E4M3", format);
    if ((uintptr_t)dev_mem & 255) return fail(CHIRON_ERR_INVALID_ARG, "dev_mem must be 256-byte aligned");
    const uint64_t need = (uint64_t)chiron_kv8_pool_bytes(m, num_blocks);
    if (bytes < need)
        return fail(CHIRON_ERR_OOM, "pool of %d pages: %llu bytes given, %llu needed", num_blocks, (unsigned long long)bytes, (unsigned long long)need);
    chiron_kvpool8* p = new (std::nothrow) chiron_kvpool8();
    if (!p) return fail(CHIRON_ERR_OOM, "host allocation failed");
    p->d = pool8_layout(m, num_blocks);
    p->d.base = (uint8_t*)dev_mem;
    p->d.format = format;
    *out = p;
    return CHIRON_OK;
}

int32_t chiron_kv8_pool_destroy(chiron_kvpool8* p) {
    delete p;
    return CHIRON_OK;
}

int32_t chiron_kv8_append_rope(chiron_kvpool8* p, int32_t layer, const chiron_new_rows* in, const int32_t* block_table, int32_t max_blocks_per_seq,
                               const int32_t* row_starts, const int32_t* seq_lens, int32_t batch, int32_t rows, void* stream) {
    if (!p || !in) return fail(CHIRON_ERR_INVALID_ARG, "pool or rows is null");
    if (layer < 0 || layer >= p->d.n_layers) return fail(CHIRON_ERR_INVALID_ARG, "layer %d out of range", layer);
    Append8Args a;
    a.pool = p->d;
    bool nothing, vec;
    int64_t wgs;
    int32_t rc = new_row_args(in, p->d.n_kv, p->d.d, layer, block_table, max_blocks_per_seq, row_starts, seq_lens, batch, rows, a, nothing, wgs, vec);
    if (rc || nothing) return rc;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)wgs);
    const bool f32 = in->dtype == CHIRON_F32;
#define CHIRON_APPEND8(D_, FMT_)                                                                      \
    do {                                                                                              \
        if (f32 && vec) launch(append8_rope_kernel<D_, FMT_, true, true>, grid, dim3(256), st, a);    \
        else if (f32) launch(append8_rope_kernel<D_, FMT_, true, false>, grid, dim3(256), st, a);     \
        else if (vec) launch(append8_rope_kernel<D_, FMT_, false, true>, grid, dim3(256), st, a);     \
        else launch(append8_rope_kernel<D_, FMT_, false, false>, grid, dim3(256), st, a);             \
    } while (0)
    const bool int8 = p->d.format == CHIRON_INT8;
    if (p->d.d == 128 && int8) CHIRON_APPEND8(128, kFmtInt8);
    else if (p->d.d == 128) CHIRON_APPEND8(128, kFmtE4m3);
    else if (int8) CHIRON_APPEND8(64, kFmtInt8);
    else CHIRON_APPEND8(64, kFmtE4m3);
#undef CHIRON_APPEND8
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

int32_t chiron_kv8_gather(const chiron_kvpool8* p, int32_t layer, const int32_t* block_table, int32_t max_blocks_per_seq, const int32_t* seq_idx,
                          const int32_t* pos, int64_t n, void* k_out, void* v_out, void* stream) {
    if (!p) return fail(CHIRON_ERR_INVALID_ARG, "pool is null");
    if (layer < 0 || layer >= p->d.n_layers) return fail(CHIRON_ERR_INVALID_ARG, "layer %d out of range", layer);
    if (n < 0) return fail(CHIRON_ERR_INVALID_ARG, "n is negative");
    if (n == 0) return CHIRON_OK;
    if (!block_table || !seq_idx || !pos || !k_out || !v_out) return fail(CHIRON_ERR_INVALID_ARG, "gather: a pointer argument is null");
    if (max_blocks_per_seq < 1) return fail(CHIRON_ERR_INVALID_ARG, "max_blocks_per_seq must be positive");
    if (((uintptr_t)k_out | (uintptr_t)v_out) & 7) return fail(CHIRON_ERR_INVALID_ARG, "gather: k_out and v_out must be 8-byte aligned");
    const int64_t per = (int64_t)p->d.n_kv * (p->d.d / 16);
    if (n > ((int64_t)0x7fffffff * 256 - 255) / per) return fail(CHIRON_ERR_SHAPE, "gather: %lld tokens are too many for one call", (long long)n);
    const dim3 grid((unsigned)((n * per + 255) / 256));
    hipStream_t st = (hipStream_t)stream;
    if (p->d.format == CHIRON_INT8)
        launch(gather8_kernel<kFmtInt8>, grid, dim3(256), st, p->d, layer, block_table, max_blocks_per_seq, seq_idx, pos, n, (uint16_t*)k_out, (uint16_t*)v_out);
    else
        launch(gather8_kernel<kFmtE4m3>, grid, dim3(256), st, p->d, layer, block_table, max_blocks_per_seq, seq_idx, pos, n, (uint16_t*)k_out, (uint16_t*)v_out);
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

}  // extern "C"
