// Rotate-and-append of new tokens into the paged cache, and the page index that block selection reads.  gfx950, wave64.
//
// What a page is to both: 16 tokens x d of one KV head.  A wave owns one (page, KV head), so that it holds everything a record of the
// index needs (old tokens of the page come from the pool) and can write V, which lies transposed inside its tile, in whole 16-byte
// pieces.  Requests are ragged and the host knows neither their lengths nor where they start, so the grid has a slot for the most
// pages that `rows` tokens of `batch` requests can touch: n tokens touch at most n/16 + 2 pages, so request i owns the slots from
// row_starts[i]/16 + 2i on, and a wave finds its request by counting those whose slots have begun, 64 at a time.
//
// Bound by its bytes, of which more are written than read: 5003 bf16 rows of 32 + 2 * 8 heads of 128, which the caches do not hold, 33 us
// (5.0 TB/s), 16384 fp32 rows with the index 130 us (5.8 TB/s; a copy of 4 GiB 4.7).  64 rows 5.4 us: the launch and a chain of loads
// (where the request's rows start, its length, its pages, its rows); with the index 9.8, the old tokens' keys being one load more
// behind these.
#include <new>

#include "append_rows.h"
#include "kv_layout.h"

namespace chiron {

constexpr float kTopBf16 = 3.3895313892515355e38f;

IndexDesc index_layout(const PoolDesc& p) {
    IndexDesc x;
    x.num_blocks = p.num_blocks;
    x.n_kv = p.n_kv;
    x.d = p.d;
    x.n_layers = p.n_layers;
    const int64_t records = (int64_t)p.num_blocks * p.n_kv;
    x.exps_at = records * 2 * p.d;
    x.layer_stride = (x.exps_at + records + 255) / 256 * 256;
    return x;
}

// The record of a page: lane = (token t = lane % 16, group g = lane / 16) holds the keys of the pieces g, g + 4, ... of 8 dims of its
// token (P pieces); `live`: the page holds that token.  Maximum and minimum over the 16 tokens by rotations within the 16 lanes.
template <int P>
__device__ __forceinline__ void write_record(const IndexDesc& x, int layer, int block, int kvh, const float (&k)[P][8], bool live) {
    const int lane = threadIdx.x & 63, t = lane & 15, g = lane >> 4;
    float hi[P][8], lo[P][8], top = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = finite_or(k[p][i], kTopBf16);
            float h = live ? v : -INFINITY, l = live ? v : INFINITY;
            h = fmaxf(h, row_move<kRor8>(h)); l = fminf(l, row_move<kRor8>(l));
            h = fmaxf(h, row_move<kRor4>(h)); l = fminf(l, row_move<kRor4>(l));
            h = fmaxf(h, row_move<kRor2>(h)); l = fminf(l, row_move<kRor2>(l));
            h = fmaxf(h, row_move<kRor1>(h)); l = fminf(l, row_move<kRor1>(l));
            hi[p][i] = h;
            lo[p][i] = l;
            top = fmaxf(top, fmaxf(fabsf(h), fabsf(l)));
        }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const int e = power_of(top);
    const float up = two_to(-e);
    int8_t* codes = index_codes(x, layer, block, kvh);
    if (t == 0) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            uint32_t h[2] = {0, 0}, l[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[i / 4] |= (uint32_t)((int)ceilf(hi[p][i] * up) & 0xff) << (i % 4 * 8);
                l[i / 4] |= (uint32_t)((int)floorf(lo[p][i] * up) & 0xff) << (i % 4 * 8);
            }
            *reinterpret_cast<uint2*>(codes + (g + 4 * p) * 8) = make_uint2(h[0], h[1]);
            *reinterpret_cast<uint2*>(codes + x.d + (g + 4 * p) * 8) = make_uint2(l[0], l[1]);
        }
    }
    if (lane == 0) *index_exp(x, layer, block, kvh) = (int8_t)e;
}

struct AppendArgs : NewRowArgs {
    PoolDesc pool;
    IndexDesc index;  // base null: none
};

// workgroups 0 .. page_wgs-1: four (page slot, KV head) each; the others: queries
template <int D, bool F32, bool VEC>
__global__ __launch_bounds__(256) void append_rope_kernel(AppendArgs a) {
    constexpr int P = D / 32, H = D / 64;  // pieces of 8 dims per lane; a piece's rotary partner is H pieces further
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
    const int r0 = np.r0, r1 = np.r1, t0 = np.t0, t1 = np.t1, block = np.block;
    const int64_t row0 = np.row0;
    uint16_t* tile = a.pool.base + tile_base(a.pool, a.layer, block, kvh);

    // Everything new that the page needs is on its way before the first of it is used: rows outside the request are replaced by its first
    // or last, so that no load hangs on a branch.
    // V: lane = (dim l of 16, four tokens 4u ..); a piece holds those tokens of the dims 32b + l and 32b + 16 + l
    const int l = lane & 15, u = lane >> 4;
    float vx[D / 32][2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const void* src = (const char*)a.v + min(max(row0 + 4 * u + i, (int64_t)r0), (int64_t)r1 - 1) * a.v_stride;
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            vx[b][0][i] = load1<F32>(src, kvh * D + 32 * b + l);
            vx[b][1][i] = load1<F32>(src, kvh * D + 32 * b + 16 + l);
        }
    }
    // K: lane = (token, group); piece c of 8 dims at (c*16 + token)*8
    const int t = lane & 15, g = lane >> 4;
    const bool is_new = t >= t0 && t < t1;
    const int64_t r = min(max(row0 + t, (int64_t)r0), (int64_t)r1 - 1);
    float kx[H][8], ky[H][8], kc[H][8], ks[H][8];
#pragma unroll
    for (int p = 0; p < H; ++p) {
        const int e = (g + 4 * p) * 8;
        const void* src = (const char*)a.k + r * a.k_stride;
        load8<F32, VEC>(src, kvh * D + e, kx[p]);
        load8<F32, VEC>(src, kvh * D + e + D / 2, ky[p]);
        load8<true, true>(a.cos_t + r * (D / 2), e, kc[p]);
        load8<true, true>(a.sin_t + r * (D / 2), e, ks[p]);
    }
    float k[P][8];
    if (is_new) {
#pragma unroll
        for (int p = 0; p < H; ++p) {
            uint4 ux, uy;
            uint32_t *px = &ux.x, *py = &uy.x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Turned w0 = turn(kx[p][2 * i], ky[p][2 * i], kc[p][2 * i], ks[p][2 * i]);
                const Turned w1 = turn(kx[p][2 * i + 1], ky[p][2 * i + 1], kc[p][2 * i + 1], ks[p][2 * i + 1]);
                px[i] = pack_bf16_rne(w0.a, w1.a);
                py[i] = pack_bf16_rne(w0.b, w1.b);
                k[p][2 * i] = bf16_lo(px[i]);
                k[p][2 * i + 1] = bf16_hi(px[i]);
                k[p + H][2 * i] = bf16_lo(py[i]);
                k[p + H][2 * i + 1] = bf16_hi(py[i]);
            }
            *reinterpret_cast<uint4*>(tile + ((g + 4 * p) * 16 + t) * 8) = ux;
            *reinterpret_cast<uint4*>(tile + ((g + 4 * (p + H)) * 16 + t) * 8) = uy;
        }
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (a.index.base && t < t0) load8<false, true>(tile, ((g + 4 * p) * 16 + t) * 8, k[p]);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) k[p][i] = 0.f;
    }
    if (a.index.base) write_record<P>(a.index, a.layer, block, kvh, k, t < t1);

    uint16_t* vtile = tile + 16 * D;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
        const float (&x)[2][4] = vx[b];
        const uint4 w = make_uint4(pack_bf16_rne(x[0][0], x[0][1]), pack_bf16_rne(x[0][2], x[0][3]), pack_bf16_rne(x[1][0], x[1][1]),
                                   pack_bf16_rne(x[1][2], x[1][3]));
        uint16_t* dst = vtile + ((b * 4 + u) * 16 + l) * 8;
        if (4 * u >= t0 && 4 * u + 4 <= t1) *reinterpret_cast<uint4*>(dst) = w;
        else {
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (4 * u + i >= t0 && 4 * u + i < t1) {
                    dst[i] = (uint16_t)(words[i / 2] >> (i % 2 * 16));
                    dst[4 + i] = (uint16_t)(words[2 + i / 2] >> (i % 2 * 16));
                }
        }
    }
}

// one wave per (request and page behind from[i]/16, KV head, layer)
template <int D>
__global__ __launch_bounds__(256) void index_update_kernel(PoolDesc pool, IndexDesc x, int layer0, const int32_t* __restrict__ bt,
                                                           int max_blocks, const int32_t* __restrict__ from, const int32_t* __restrict__ to,
                                                           int batch, int pages) {
    constexpr int P = D / 32;
    const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int kvh = (int)(task % pool.n_kv);
    const int64_t slot = task / pool.n_kv;
    const int req = (int)(slot / pages), layer = layer0 + blockIdx.y;
    if (req >= batch) return;
    const int f = from[req], end = to[req];
    if (f < 0 || end <= f) return;
    const int page = f / kBlockSize + (int)(slot % pages);
    if (page >= max_blocks || (int64_t)page * kBlockSize >= end) return;
    const int block = bt[(size_t)req * max_blocks + page];
    if (block < 0 || block >= pool.num_blocks) return;
    const int lane = threadIdx.x & 63, t = lane & 15, g = lane >> 4;
    const bool live = (int64_t)page * kBlockSize + t < end;
    const uint16_t* tile = pool.base + tile_base(pool, layer, block, kvh);
    float k[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p) load8<false, true>(tile, ((g + 4 * p) * 16 + t) * 8, k[p]);
    write_record<P>(x, layer, block, kvh, k, live);
}

}  // namespace chiron

using namespace chiron;

extern "C" {

int64_t chiron_kv_index_bytes(const chiron_kvpool* p) {
    if (!p) return 0;
    const IndexDesc x = index_layout(p->d);
    return x.layer_stride * x.n_layers;
}

int32_t chiron_kv_index_create(const chiron_kvpool* p, void* dev_mem, uint64_t bytes, chiron_kvindex** out) {
    if (!out) return fail(CHIRON_ERR_INVALID_ARG, "out is null");
    *out = nullptr;
    if (!p || !dev_mem) return fail(CHIRON_ERR_INVALID_ARG, "pool or dev_mem is null");
    if ((uintptr_t)dev_mem & 255) return fail(CHIRON_ERR_INVALID_ARG, "dev_mem must be 256-byte aligned");
    const uint64_t need = (uint64_t)chiron_kv_index_bytes(p);
    if (bytes < need) return fail(CHIRON_ERR_OOM, "page index: %llu bytes given, %llu needed", (unsigned long long)bytes, (unsigned long long)need);
    chiron_kvindex* x = new (std::nothrow) chiron_kvindex();
    if (!x) return fail(CHIRON_ERR_OOM, "host allocation failed");
    x->d = index_layout(p->d);
    x->d.base = (int8_t*)dev_mem;
    *out = x;
    return CHIRON_OK;
}

int32_t chiron_kv_index_destroy(chiron_kvindex* x) {
    delete x;
    return CHIRON_OK;
}

int32_t chiron_kv_index_update(chiron_kvindex* x, const chiron_kvpool* p, int32_t layer, int32_t n_layers, const int32_t* block_table,
                               int32_t max_blocks_per_seq, const int32_t* from, const int32_t* to, int32_t batch, int32_t max_new,
                               void* stream) {
    if (!x || !p) return fail(CHIRON_ERR_INVALID_ARG, "index or pool is null");
    if (!index_fits(x->d, p->d)) return fail(CHIRON_ERR_INVALID_ARG, "the page index was created for another pool shape");
    if (batch < 0 || max_new < 0 || n_layers < 0) return fail(CHIRON_ERR_INVALID_ARG, "index update: a size is negative");
    if (layer < 0 || n_layers > p->d.n_layers - layer) return fail(CHIRON_ERR_INVALID_ARG, "layers %d .. %lld are out of range", layer, (long long)layer + n_layers - 1);
    if (batch == 0 || max_new == 0 || n_layers == 0) return CHIRON_OK;
    if (!block_table || !from || !to) return fail(CHIRON_ERR_INVALID_ARG, "index update: a pointer argument is null");
    if (max_blocks_per_seq < 1) return fail(CHIRON_ERR_INVALID_ARG, "max_blocks_per_seq must be positive");
    const int64_t pages64 = ((int64_t)max_new + 14) / kBlockSize + 1;
    const int pages = (int)(pages64 < max_blocks_per_seq ? pages64 : max_blocks_per_seq);
    const int64_t wgs = ((int64_t)batch * pages * p->d.n_kv + 3) / 4;
    if (wgs > 0x7fffffff || n_layers > 65535) return fail(CHIRON_ERR_SHAPE, "index update: %lld pages at once are too many", (long long)batch * pages);
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)wgs, n_layers);
    if (p->d.d == 128) launch(index_update_kernel<128>, grid, dim3(256), st, p->d, x->d, layer, block_table, max_blocks_per_seq, from, to, batch, pages);
    else launch(index_update_kernel<64>, grid, dim3(256), st, p->d, x->d, layer, block_table, max_blocks_per_seq, from, to, batch, pages);
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

int32_t chiron_append_kv_rope(chiron_kvpool* p, chiron_kvindex* index, int32_t layer, const chiron_new_rows* in, const int32_t* block_table,
                              int32_t max_blocks_per_seq, const int32_t* row_starts, const int32_t* seq_lens, int32_t batch, int32_t rows,
                              void* stream) {
    if (!p || !in) return fail(CHIRON_ERR_INVALID_ARG, "pool or rows is null");
    if (layer < 0 || layer >= p->d.n_layers) return fail(CHIRON_ERR_INVALID_ARG, "layer %d out of range", layer);
    if (index && !index_fits(index->d, p->d)) return fail(CHIRON_ERR_INVALID_ARG, "the page index was created for another pool shape");
    AppendArgs a;
    a.pool = p->d;
    if (index) a.index = index->d;
    bool nothing, vec;
    int64_t wgs;
    int32_t rc = new_row_args(in, p->d.n_kv, p->d.d, layer, block_table, max_blocks_per_seq, row_starts, seq_lens, batch, rows, a, nothing, wgs, vec);
    if (rc || nothing) return rc;
    const int d = p->d.d;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)wgs);
    const bool f32 = in->dtype == CHIRON_F32;
#define CHIRON_APPEND(D_)                                                                        \
    do {                                                                                         \
        if (f32 && vec) launch(append_rope_kernel<D_, true, true>, grid, dim3(256), st, a);      \
        else if (f32) launch(append_rope_kernel<D_, true, false>, grid, dim3(256), st, a);       \
        else if (vec) launch(append_rope_kernel<D_, false, true>, grid, dim3(256), st, a);       \
        else launch(append_rope_kernel<D_, false, false>, grid, dim3(256), st, a);               \
    } while (0)
    if (d == 128) CHIRON_APPEND(128);
    else CHIRON_APPEND(64);
#undef CHIRON_APPEND
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

int32_t chiron_op_rope_table(const int32_t* pos, int32_t rows, int32_t d, float base, float* cos, float* sin, void* stream) {
    if (rows < 0 || d < 2 || (d & 1)) return fail(CHIRON_ERR_INVALID_ARG, "rope table: bad sizes");
    if (!(base > 1.0f)) return fail(CHIRON_ERR_INVALID_ARG, "rope table: base must be > 1");
    if (rows == 0) return CHIRON_OK;
    if (!pos || !cos || !sin) return fail(CHIRON_ERR_INVALID_ARG, "rope table: a pointer is null");
    if ((int64_t)rows * (d / 2) > 0x7fffffff) return fail(CHIRON_ERR_SHAPE, "rope table: rows*d/2 = %lld exceeds 2^31-1", (long long)rows * (d / 2));
    return launch_rope_table(pos, rows, d, base, cos, sin, (hipStream_t)stream);
}

}  // extern "C"
