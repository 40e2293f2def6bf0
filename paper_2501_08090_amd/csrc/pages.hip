// Page lists: block tables and slot maps from request lengths, on the device.  gfx950, wave64.
//
// Whole numbers in a fixed order: a request's place in the list and its rows follow from sums over the requests before it.  Where the table
// is small one workgroup does everything in one launch, with the sums by data-parallel scans over its waves; larger ones take a launch
// for the counts (a wave per request), one for the sums (one workgroup) and one or two that write.
#include <algorithm>

#include "chiron_internal.h"
#include "device_util.h"

namespace chiron {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / 64;

// sums over the workgroup of a pair of 64-bit values, thread by thread: `incl` gets the sums up to and with this thread's, the return
// value those over all
struct Pair {
    int64_t a, b;
};
__device__ __forceinline__ Pair wave_scan(Pair v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t a = __shfl_up(v.a, o), b = __shfl_up(v.b, o);
        if (lane >= o) {
            v.a += a;
            v.b += b;
        }
    }
    return v;
}
__device__ __forceinline__ Pair block_scan(Pair v, Pair* lds /* [kPageWaves] */, Pair& incl) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    incl = wave_scan(v);
    __syncthreads();
    if (lane == 63) lds[wave] = incl;
    __syncthreads();
    Pair all{0, 0};
#pragma unroll
    for (int w = 0; w < kPageWaves; ++w) {
        const Pair x = lds[w];
        if (w < wave) {
            incl.a += x.a;
            incl.b += x.b;
        }
        all.a += x.a;
        all.b += x.b;
    }
    return all;
}

// ---- what both need: columns [c0, c1) of a request's table row, of which those are counted and written that hold a page (release) or hold
// none (grant)
struct PageArgs {
    int32_t *list, *count;
    int capacity;
    int32_t* bt;
    int width, batch, max_rows;
    const int32_t *first, *second;  // release: from, to (may be null); grant: seq_lens, new_lens
    int32_t *row_starts, *row_seq, *pos, *granted;
    int64_t* slots;
    int32_t *need, *at;  // workspace: per request how many columns count, and the place in the list that goes with the first of them
};
template <bool GRANT>
__device__ __forceinline__ void columns(const PageArgs& a, int i, int& c0, int& c1) {
    if (GRANT) {
        const int64_t old = a.first[i], n = a.second[i];
        const bool fits = old >= 0 && n > 0 && old + n <= (int64_t)a.width * kBlockSize;
        c0 = fits ? (int)(old / kBlockSize) : 0;
        c1 = fits ? (int)((old + n - 1) / kBlockSize) + 1 : 0;
    } else {
        c0 = (int)min(((int64_t)max(a.first[i], 0) + kBlockSize - 1) / kBlockSize, (int64_t)a.width);
        c1 = a.second ? min(max(a.second[i], 0) / kBlockSize, a.width) : a.width;
    }
}
template <bool GRANT>
__device__ __forceinline__ bool counts(int entry) {
    return GRANT ? entry < 0 : entry >= 0;
}
// by a whole wave: how many columns of request i count
template <bool GRANT>
__device__ __forceinline__ int count_columns(const PageArgs& a, int i) {
    int c0, c1;
    columns<GRANT>(a, i, c0, c1);
    const int32_t* row = a.bt + (size_t)i * a.width;
    const int lane = threadIdx.x & 63;
    int n = 0;
    constexpr int kAtOnce = 8;  // loads on their way together
    for (int c = c0; c < c1; c += 64 * kAtOnce) {
        int e[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int j = c + 64 * u + lane;
            e[u] = j < c1 ? row[j] : GRANT ? 0 : -1;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) n += __popcll(__ballot(counts<GRANT>(e[u])));
    }
    return n;
}
// one of them: list[k] goes to a column, or a column's page to list[k]
template <bool GRANT>
__device__ __forceinline__ void move_page(const PageArgs& a, int32_t* entry, int page, int k) {
    if (k < 0 || k >= a.capacity) return;
    if (GRANT) *entry = a.list[k];
    else {
        a.list[k] = page;
        *entry = -1;
    }
}
// by a whole wave: those columns get the pages list[at ..] (grant), or their pages go to list[at ..] (release)
template <bool GRANT>
__device__ __forceinline__ void move_pages(const PageArgs& a, int i, int at) {
    int c0, c1;
    columns<GRANT>(a, i, c0, c1);
    int32_t* row = a.bt + (size_t)i * a.width;
    const int lane = threadIdx.x & 63;
    constexpr int kAtOnce = 4;
    for (int c = c0; c < c1; c += 64 * kAtOnce) {
        int e[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int j = c + 64 * u + lane;
            e[u] = j < c1 ? row[j] : GRANT ? 0 : -1;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const bool mine = counts<GRANT>(e[u]);
            const uint64_t all = __ballot(mine);
            const int k = at + __popcll(all & (((uint64_t)1 << lane) - 1));
            if (mine) move_page<GRANT>(a, row + c + 64 * u + lane, e[u], k);
            at += __popcll(all);
        }
    }
}

// The sums, by one workgroup; need[] of every request is there.
__device__ __forceinline__ void grant_sums(const PageArgs& a, Pair* lds) {
    const int64_t there = min(max(*a.count, 0), a.capacity);
    const int64_t table = (int64_t)a.width * kBlockSize;
    Pair before{0, 0}, given{0, 0};  // (rows, pages): of all requests that fit, of those granted
    for (int i0 = 0; i0 < a.batch; i0 += kPageThreads) {
        const int i = i0 + threadIdx.x;
        int64_t n = 0, need = 0;
        if (i < a.batch) {
            const int64_t old = a.first[i];
            n = a.second[i];
            if (old < 0 || n < 0 || old + n > table) n = 0;
            need = n > 0 ? a.need[i] : 0;
        }
        Pair incl;
        const Pair all = block_scan(Pair{n, need}, lds, incl);
        const bool ok = before.a + incl.a <= a.max_rows && (need == 0 || before.b + incl.b <= there);
        before.a += all.a;
        before.b += all.b;
        const Pair all2 = block_scan(Pair{ok ? n : 0, ok ? need : 0}, lds, incl);
        if (i < a.batch) {
            a.row_starts[i + 1] = (int32_t)(given.a + incl.a);
            if (a.granted) a.granted[i] = ok ? (int32_t)n : 0;
            a.need[i] = ok ? (int32_t)need : 0;
            a.at[i] = (int32_t)(given.b + incl.b - need);  // counted from the first page taken, which is not known yet
        }
        given.a += all2.a;
        given.b += all2.b;
    }
    const int32_t left = (int32_t)(there - given.b);
    for (int i = threadIdx.x; i < a.batch; i += kPageThreads) a.at[i] += left;  // the thread's own words
    if (threadIdx.x == 0) {
        a.row_starts[0] = 0;
        *a.count = left;
    }
}
__device__ __forceinline__ void release_sums(const PageArgs& a, Pair* lds) {
    const int64_t there = min(max(*a.count, 0), a.capacity);
    int64_t before = 0;
    for (int i0 = 0; i0 < a.batch; i0 += kPageThreads) {
        const int i = i0 + threadIdx.x;
        const int64_t n = i < a.batch ? a.need[i] : 0;
        Pair incl;
        const Pair all = block_scan(Pair{n, 0}, lds, incl);
        if (i < a.batch) a.at[i] = (int32_t)min(there + before + incl.a - n, (int64_t)a.capacity);
        before += all.a;
    }
    __syncthreads();  // every wave has read the count
    if (threadIdx.x == 0) *a.count = (int32_t)min(there + before, (int64_t)a.capacity);
}

// rows r0 .. r0+255 by 256 threads
__device__ __forceinline__ void write_rows(const PageArgs& a, int64_t r0, int tid) {
    const int64_t r = r0 + tid;
    if (r >= a.max_rows) return;
    // the last request whose rows begin at or before r: those without rows begin where the next one does
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.row_starts[mid] <= r) lo = mid;
        else hi = mid;
    }
    const bool live = a.batch > 0 && r < a.row_starts[a.batch];
    int64_t slot = -1;
    int pos = 0;
    if (live) {
        pos = (int)(a.first[lo] + (r - a.row_starts[lo]));
        const int page = a.bt[(size_t)lo * a.width + pos / kBlockSize];
        if (page >= 0) slot = (int64_t)page * kBlockSize + pos % kBlockSize;
    }
    if (a.row_seq) a.row_seq[r] = live ? lo : -1;
    if (a.pos) a.pos[r] = pos;
    if (a.slots) a.slots[r] = slot;
}

// Everything by one workgroup.  Requests of a few columns (a token or a few more) are a thread's, the others a wave's: one column a wave
// takes as long as 512.
constexpr int kFewColumns = 4, kOneBatch = 1024;
template <bool GRANT>
__global__ __launch_bounds__(kPageThreads) void pages_one_kernel(PageArgs a) {
    __shared__ Pair lds[kPageWaves];
    __shared__ int many[kOneBatch], n_many;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, mine = threadIdx.x;
    if (mine == 0) n_many = 0;
    __syncthreads();
    int c0 = 0, c1 = 0;
    int32_t* row = a.bt + (size_t)mine * a.width;
    if (mine < a.batch) {
        columns<GRANT>(a, mine, c0, c1);
        if (c1 - c0 > kFewColumns) many[atomicAdd(&n_many, 1)] = mine;  // in any order: each writes its own words
        else {
            int n = 0;
#pragma unroll
            for (int u = 0; u < kFewColumns; ++u) n += c0 + u < c1 && counts<GRANT>(row[c0 + u]);
            a.need[mine] = n;
        }
    }
    __syncthreads();
    for (int k = wave; k < n_many; k += kPageWaves) {
        const int n = count_columns<GRANT>(a, many[k]);
        if (lane == 0) a.need[many[k]] = n;
    }
    __syncthreads();
    if (GRANT) grant_sums(a, lds);
    else release_sums(a, lds);
    __syncthreads();
    if (mine < a.batch && c1 - c0 <= kFewColumns && a.need[mine] > 0) {
        int k = a.at[mine];
        for (int c = c0; c < c1; ++c)
            if (counts<GRANT>(row[c])) move_page<GRANT>(a, row + c, row[c], k++);
    }
    for (int k = wave; k < n_many; k += kPageWaves)
        if (a.need[many[k]] > 0) move_pages<GRANT>(a, many[k], a.at[many[k]]);
    if (GRANT) {
        __syncthreads();
        for (int64_t r0 = 0; r0 < a.max_rows; r0 += kPageThreads) write_rows(a, r0, threadIdx.x);
    }
}

template <bool GRANT>
__global__ __launch_bounds__(256) void pages_count_kernel(PageArgs a) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= a.batch) return;
    const int n = count_columns<GRANT>(a, i);
    if ((threadIdx.x & 63) == 0) a.need[i] = n;
}
template <bool GRANT>
__global__ __launch_bounds__(kPageThreads) void pages_sums_kernel(PageArgs a) {
    __shared__ Pair lds[kPageWaves];
    if (GRANT) grant_sums(a, lds);
    else release_sums(a, lds);
}
template <bool GRANT>
__global__ __launch_bounds__(256) void pages_move_kernel(PageArgs a) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i < a.batch && a.need[i] > 0) move_pages<GRANT>(a, i, a.at[i]);
}
__global__ __launch_bounds__(256) void pages_rows_kernel(PageArgs a) { write_rows(a, (int64_t)blockIdx.x * 256, threadIdx.x); }

static int32_t check_list(const chiron_page_list* l, int32_t batch, int32_t width) {
    if (!l) return fail(CHIRON_ERR_INVALID_ARG, "page list is null");
    if (l->capacity > 1 << 30) return fail(CHIRON_ERR_SHAPE, "pages: a list of %d pages is too long", l->capacity);
    if (batch < 0 || l->capacity < 0) return fail(CHIRON_ERR_INVALID_ARG, "pages: a size is negative");
    if (width < 1 || width > 1 << 26) return fail(CHIRON_ERR_INVALID_ARG, "pages: max_blocks_per_seq %d is not in 1 .. 2^26", width);
    if (!l->count || (!l->pages && l->capacity > 0)) return fail(CHIRON_ERR_INVALID_ARG, "pages: a pointer of the list is null");
    return CHIRON_OK;
}
static PageArgs page_args(const chiron_page_list* l, int32_t* bt, int32_t width, const int32_t* first, const int32_t* second, int32_t batch,
                          void* workspace) {
    PageArgs a = {};
    a.list = l->pages; a.count = l->count; a.capacity = l->capacity;
    a.bt = bt; a.width = width; a.batch = batch; a.first = first; a.second = second;
    a.need = (int32_t*)workspace; a.at = a.need + batch;
    return a;
}

}  // namespace chiron

using namespace chiron;

extern "C" {

int64_t chiron_kv_pages_workspace_bytes(int32_t batch) { return batch < 0 ? 0 : 16 + (8 * (int64_t)batch + 15) / 16 * 16; }

int32_t chiron_kv_grant_pages(const chiron_page_list* list, int32_t* block_table, int32_t max_blocks_per_seq, const int32_t* seq_lens,
                              const int32_t* new_lens, int32_t batch, int32_t max_rows, const chiron_row_maps* out, void* workspace,
                              void* stream) {
    int32_t rc = check_list(list, batch, max_blocks_per_seq);
    if (rc) return rc;
    if (max_rows < 0) return fail(CHIRON_ERR_INVALID_ARG, "pages: a size is negative");
    if (!out || !out->row_starts) return fail(CHIRON_ERR_INVALID_ARG, "pages: row_starts is null");
    if (!workspace || ((uintptr_t)workspace & 15)) return fail(CHIRON_ERR_INVALID_ARG, "pages: the workspace is null or not 16-byte aligned");
    if (batch > 0 && (!block_table || !seq_lens || !new_lens)) return fail(CHIRON_ERR_INVALID_ARG, "pages: a pointer argument is null");
    PageArgs a = page_args(list, block_table, max_blocks_per_seq, seq_lens, new_lens, batch, workspace);
    a.max_rows = max_rows;
    a.row_starts = out->row_starts; a.row_seq = out->row_seq; a.pos = out->pos; a.granted = out->granted; a.slots = out->slots;
    hipStream_t st = (hipStream_t)stream;
    const bool rows = out->row_seq || out->pos || out->slots;
    if (batch <= kOneBatch && max_rows <= 8192) {
        launch(pages_one_kernel<true>, dim3(1), dim3(kPageThreads), st, a);
    } else {
        const dim3 waves((unsigned)((batch + 3) / 4));
        if (batch) launch(pages_count_kernel<true>, waves, dim3(256), st, a);
        launch(pages_sums_kernel<true>, dim3(1), dim3(kPageThreads), st, a);
        if (batch) launch(pages_move_kernel<true>, waves, dim3(256), st, a);
        if (rows && max_rows) launch(pages_rows_kernel, dim3((unsigned)(((int64_t)max_rows + 255) / 256)), dim3(256), st, a);
    }
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

int32_t chiron_kv_release_pages(const chiron_page_list* list, int32_t* block_table, int32_t max_blocks_per_seq, const int32_t* from,
                                const int32_t* to, int32_t batch, void* workspace, void* stream) {
    int32_t rc = check_list(list, batch, max_blocks_per_seq);
    if (rc) return rc;
    if (!workspace || ((uintptr_t)workspace & 15)) return fail(CHIRON_ERR_INVALID_ARG, "pages: the workspace is null or not 16-byte aligned");
    if (batch == 0) return CHIRON_OK;
    if (!block_table || !from) return fail(CHIRON_ERR_INVALID_ARG, "pages: a pointer argument is null");
    const PageArgs a = page_args(list, block_table, max_blocks_per_seq, from, to, batch, workspace);
    hipStream_t st = (hipStream_t)stream;
    if ((int64_t)batch * max_blocks_per_seq <= 65536 && batch <= kOneBatch) {
        launch(pages_one_kernel<false>, dim3(1), dim3(kPageThreads), st, a);
    } else {
        const dim3 waves((unsigned)((batch + 3) / 4));
        launch(pages_count_kernel<false>, waves, dim3(256), st, a);
        launch(pages_sums_kernel<false>, dim3(1), dim3(kPageThreads), st, a);
        launch(pages_move_kernel<false>, waves, dim3(256), st, a);
    }
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

}  // extern "C"
