// What every append of new rows shares: loading rows of fp32 or bf16, the rotation, finding the page that a wave writes, rotating the
// queries, and the checks of the arguments.
#pragma once

#include "draft_ops.h"

namespace chiron {

// 4 values from dim e on of a row of fp32 or bf16; VEC: 16-byte aligned; STREAM: nobody reads them again
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <bool F32, bool VEC, bool STREAM>
__device__ __forceinline__ void load4(const void* row, int e, float (&x)[4]) {
    if (F32) {
        const float* p = reinterpret_cast<const float*>(row) + e;
        if (VEC) {
            const floatx4* pv = reinterpret_cast<const floatx4*>(p);
            const floatx4 a = STREAM ? __builtin_nontemporal_load(pv) : *pv;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = a[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = p[i];
        }
    } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + e;
        if (VEC) {
            const u32x2* pv = reinterpret_cast<const u32x2*>(p);
            const u32x2 a = STREAM ? __builtin_nontemporal_load(pv) : *pv;
            x[0] = bf16_lo(a[0]); x[1] = bf16_hi(a[0]); x[2] = bf16_lo(a[1]); x[3] = bf16_hi(a[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __uint_as_float((uint32_t)p[i] << 16);
        }
    }
}
// 8
template <bool F32, bool VEC>
__device__ __forceinline__ void load8(const void* row, int e, float (&x)[8]) {
    if (F32) {
        const float* p = reinterpret_cast<const float*>(row) + e;
        if (VEC) {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[i];
        }
    } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + e;
        if (VEC) {
            const uint4 a = *reinterpret_cast<const uint4*>(p);
            x[0] = bf16_lo(a.x); x[1] = bf16_hi(a.x); x[2] = bf16_lo(a.y); x[3] = bf16_hi(a.y);
            x[4] = bf16_lo(a.z); x[5] = bf16_hi(a.z); x[6] = bf16_lo(a.w); x[7] = bf16_hi(a.w);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((uint32_t)p[i] << 16);
        }
    }
}
template <bool F32>
__device__ __forceinline__ float load1(const void* row, int e) {
    return F32 ? reinterpret_cast<const float*>(row)[e] : __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(row)[e] << 16);
}

// One pair of the rotation.  The products are rounded one by one, not fused into the sum: what is stored, and the index record that
// follows from it, is then the same as elementary fp32 operations give.
struct Turned {
    float a, b;
};
__device__ __forceinline__ Turned turn(float x, float y, float c, float s) {
#pragma clang fp contract(off)
    const float xc = x * c, ys = y * s, yc = y * c, xs = x * s;
    return Turned{xc - ys, yc + xs};
}

struct NewRowArgs {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;  // bytes
    const float *cos_t, *sin_t;
    float* q_out;
    const int32_t *bt, *row_starts, *seq_lens;
    int layer, n_q, max_blocks, batch, rows, page_wgs;
    bool stream;  // the queries with the streaming hint
};

// 4 dims of the lower half of a head and their partners, so that a wave's loads and stores are whole lines
template <int D, bool F32, bool VEC, bool STREAM>
__device__ __forceinline__ void rotate_queries(const NewRowArgs& a) {
    const int64_t j = (int64_t)(blockIdx.x - a.page_wgs) * 256 + threadIdx.x;  // (row, head, piece)
    const int per_row = a.n_q * (D / 8);
    const int64_t r = j / per_row;
    if (r >= a.rows) return;
    const int w = (int)(j - r * per_row), head = w / (D / 8), e = w % (D / 8) * 4;
    const void* src = (const char*)a.q + r * a.q_stride;
    float x[4], y[4];
    load4<F32, VEC, STREAM>(src, head * D + e, x);
    load4<F32, VEC, STREAM>(src, head * D + e + D / 2, y);
    const floatx4 c = *reinterpret_cast<const floatx4*>(a.cos_t + r * (D / 2) + e), s = *reinterpret_cast<const floatx4*>(a.sin_t + r * (D / 2) + e);
    floatx4 u, v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Turned w = turn(x[i], y[i], c[i], s[i]);
        u[i] = w.a;
        v[i] = w.b;
    }
    floatx4* dst = reinterpret_cast<floatx4*>(a.q_out + (r * a.n_q + head) * D + e);
    if (STREAM) {
        __builtin_nontemporal_store(u, dst);
        __builtin_nontemporal_store(v, dst + D / 8);
    } else {
        dst[0] = u;
        dst[D / 8] = v;
    }
}

// The page that goes with a page slot, by a whole wave: request i owns the slots from row_starts[i]/16 + 2i on.
struct NewPage {
    int r0, r1;    // the request's rows
    int block, t0, t1;  // the page in the pool, and its new tokens
    int64_t row0;  // the row of the page's token 0 (may lie before r0)
};
__device__ __forceinline__ bool new_page(const NewRowArgs& a, int slot, int num_blocks, NewPage& n) {
    const int lane = threadIdx.x & 63;
    int req = -1;  // the last i whose first slot is not behind this one
    for (int i0 = 0; i0 < a.batch; i0 += 64) {
        const int i = min(i0 + lane, a.batch - 1);
        const uint64_t begun = __ballot(i0 + lane < a.batch && a.row_starts[i] / kBlockSize + 2 * i <= slot);
        req += __popcll(begun);
        if (begun != ~(uint64_t)0) break;
    }
    if (req < 0) return false;
    const int r0 = a.row_starts[req], r1 = a.row_starts[req + 1], old = a.seq_lens[req];
    if (r0 < 0 || r1 > a.rows || r1 <= r0 || old < 0) return false;
    const int ahead = slot - (r0 / kBlockSize + 2 * req);  // below 0 only where the row starts do not ascend
    const int page = old / kBlockSize + ahead;
    const int64_t end = (int64_t)old + (r1 - r0), first = (int64_t)page * kBlockSize;
    if (ahead < 0 || first >= end || page >= a.max_blocks) return false;
    const int block = a.bt[(size_t)req * a.max_blocks + page];
    if (block < 0 || block >= num_blocks) return false;
    n.r0 = r0;
    n.r1 = r1;
    n.block = block;
    n.t0 = (int)max((int64_t)0, old - first);
    n.t1 = (int)min((int64_t)kBlockSize, end - first);
    n.row0 = r0 + first - old;
    return true;
}

inline bool aligned16(const void* p, int64_t stride_bytes) { return ((uintptr_t)p & 15) == 0 && stride_bytes % 16 == 0; }

// Checks an append's arguments and fills in the kernel's.  `nothing`: there is nothing to do; `wgs`: workgroups of 256 for page slots
// and queries; `vec`: rows can be loaded in 16-byte pieces.
inline int32_t new_row_args(const chiron_new_rows* in, int n_kv, int d, int32_t layer, const int32_t* block_table, int32_t max_blocks_per_seq,
                            const int32_t* row_starts, const int32_t* seq_lens, int32_t batch, int32_t rows, NewRowArgs& a, bool& nothing,
                            int64_t& wgs, bool& vec) {
    nothing = false;
    if (batch < 0 || rows < 0) return fail(CHIRON_ERR_INVALID_ARG, "append: a size is negative");
    if (in->dtype != CHIRON_F32 && in->dtype != CHIRON_BF16) return fail(CHIRON_ERR_INVALID_ARG, "append: dtype %d is neither CHIRON_F32 nor CHIRON_BF16", in->dtype);
    if (!in->q != !in->q_out) return fail(CHIRON_ERR_INVALID_ARG, "append: q and q_out come together");
    if (in->q && (in->n_q_heads < 1 || in->n_q_heads > 0x7fffffff / d)) return fail(CHIRON_ERR_INVALID_ARG, "append: n_q_heads %d", in->n_q_heads);
    if (rows == 0) {
        nothing = true;
        return CHIRON_OK;
    }
    if (batch == 0) return fail(CHIRON_ERR_INVALID_ARG, "append: %d rows of no request", rows);
    if (!in->k || !in->v || !in->cos || !in->sin || !block_table || !row_starts || !seq_lens)
        return fail(CHIRON_ERR_INVALID_ARG, "append: a pointer argument is null");
    if (max_blocks_per_seq < 1) return fail(CHIRON_ERR_INVALID_ARG, "max_blocks_per_seq must be positive");
    const int64_t kv_row = (int64_t)n_kv * d;
    if (in->k_stride < kv_row || in->v_stride < kv_row || (in->q && in->q_stride < (int64_t)in->n_q_heads * d))
        return fail(CHIRON_ERR_INVALID_ARG, "append: a row stride is smaller than the row");
    if (((uintptr_t)in->cos | (uintptr_t)in->sin | (uintptr_t)in->q_out) & 15)
        return fail(CHIRON_ERR_INVALID_ARG, "append: cos, sin and q_out must be 16-byte aligned");
    const int size = in->dtype == CHIRON_F32 ? 4 : 2;
    if (((uintptr_t)in->q | (uintptr_t)in->k | (uintptr_t)in->v) & (size - 1)) return fail(CHIRON_ERR_INVALID_ARG, "append: q, k or v is misaligned for its type");
    a.q = in->q; a.k = in->k; a.v = in->v;
    a.q_stride = in->q_stride * size; a.k_stride = in->k_stride * size; a.v_stride = in->v_stride * size;
    a.cos_t = in->cos; a.sin_t = in->sin; a.q_out = in->q_out;
    a.bt = block_table; a.row_starts = row_starts; a.seq_lens = seq_lens;
    a.layer = layer; a.n_q = in->n_q_heads; a.max_blocks = max_blocks_per_seq; a.batch = batch; a.rows = rows;
    const int64_t tasks = ((int64_t)rows / kBlockSize + 2 * (int64_t)batch) * n_kv;
    const int64_t q_wgs = in->q ? ((int64_t)rows * in->n_q_heads * (d / 8) + 255) / 256 : 0;
    const int64_t page_wgs = (tasks + 3) / 4;  // a wave per page slot and KV head
    if (page_wgs + q_wgs > 0x7fffffff) return fail(CHIRON_ERR_SHAPE, "append: %d rows of %d heads are too many for one call", rows, in->n_q_heads);
    a.page_wgs = (int)page_wgs;
    // Queries that the L2s do not hold together go past them.  us with the hint / without, queries written to memory that no cache holds: 2048
    // bf16 rows of 32 heads of 128 (32 MiB) 15.5 / 13.9 to 18.2, 3500 24 / 26.4, 5003 31.9 / 37.1, 16384 100 / 107; fp32 rows 5003 39 / 45.6, 16384
    // 127 / 136.  Where the last call's queries lie in the same memory the two are level up to some 8000 rows.  What the hint saves here
    // is less than what a pass over the queries behind the call takes longer, up to 12000 rows (5003 bf16 rows and the pass 67.6 / 58.5, 12000
    // 149 / 132, 16384 199 / 199).
    a.stream = (int64_t)rows * in->n_q_heads * d * 4 > (32 << 20);
    wgs = page_wgs + q_wgs;
    vec = (!in->q || aligned16(in->q, a.q_stride)) && aligned16(in->k, a.k_stride);
    return CHIRON_OK;
}

}  // namespace chiron
