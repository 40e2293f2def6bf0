// Page lists: block tables and slot maps from request lengths, on the device.  gfx950, wave64.
//
// Whole numbers in a fixed order: a request's place in the list and its rows follow from sums over the requests before it.  Where the table
// is small one workgroup does everything in one launch, with the sums by data-parallel scans over its waves; larger ones take a launch
// for the counts (a wave per request), one for the sums (one workgroup) and one or two that write.
//
// Bound by latency: the small ones are one chain of load, scan, load, store, 7.6 us for 64 requests of 512 columns that ask for a token each, and 6.3 us to
// release their pages.  1501 requests that ask for up to 6 tokens, 60 of them for prompts: 4.4 (counts), 7.6 (sums), 6.3 (pages), 5.2 us (rows), and 13 us for the
// release; the bytes that move (11 MB) would take 2.
#include <algorithm>

#include "chiron_internal.h"
#include "device_util.h"

namespace chiron {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / 64;

// Sums of a pair of whole numbers that stop at kMost: what is compared with a limit below it is compared rightly however large it is.
constexpr uint32_t kMost = 0x7fffffffu;
struct Pair {
    uint32_t a, b;
};
__device__ __forceinline__ uint32_t plus(uint32_t x, uint32_t y) { return min(x + y, kMost); }  // of two up to kMost
// over a wave, by data-parallel moves as in device_util.h's wave_scan: lane l gets the sum over the lanes 0 .. l
template <int Ctrl, int Rows>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, Ctrl, Rows, 0xf, false); }
__device__ __forceinline__ uint32_t scan(uint32_t v) {
    v = plus(v, moved<0x111, 0xf>(v));
    v = plus(v, moved<0x112, 0xf>(v));
    v = plus(v, moved<0x114, 0xf>(v));
    v = plus(v, moved<0x118, 0xf>(v));
    v = plus(v, moved<0x142, 0xa>(v));
    v = plus(v, moved<0x143, 0xc>(v));
    return v;
}
// over the workgroup: `incl` gets the sums up to and with this thread's, the return value is those over all
__device__ __forceinline__ Pair block_scan(Pair v, Pair* lds /* [kPageWaves] */, Pair& incl) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    incl = Pair{scan(v.a), scan(v.b)};
    __syncthreads();
    if (lane == 63) lds[wave] = incl;
    __syncthreads();
    Pair all{0, 0};
#pragma unroll
    for (int w = 0; w < kPageWaves; ++w) {
        const Pair x = lds[w];
        if (w < wave) incl = Pair{plus(incl.a, x.a), plus(incl.b, x.b)};
        all = Pair{plus(all.a, x.a), plus(all.b, x.b)};
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

// The sums, by one workgroup; need[] of every request is there.  starts: row_starts once more, in LDS, or null.
__device__ __forceinline__ void grant_sums(const PageArgs& a, Pair* lds, int32_t* starts) {
    const uint32_t there = min(max(*a.count, 0), a.capacity);
    const int64_t table = (int64_t)a.width * kBlockSize;
    Pair before{0, 0};  // (rows, pages) of the requests so far that fit the table
    uint32_t rows = 0, pages = 0;  // of those granted
    for (int i0 = 0; i0 < a.batch; i0 += kPageThreads) {
        const int i = i0 + threadIdx.x;
        uint32_t n = 0, need = 0;
        if (i < a.batch) {
            const int64_t old = a.first[i], want = a.second[i];
            if (old >= 0 && want > 0 && old + want <= table) {
                n = (uint32_t)want;
                need = a.need[i];
            }
        }
        Pair incl;
        const Pair all = block_scan(Pair{n, need}, lds, incl);
        const bool ok = plus(before.a, incl.a) <= (uint32_t)a.max_rows && (need == 0 || plus(before.b, incl.b) <= there);
        before = Pair{plus(before.a, all.a), plus(before.b, all.b)};
        if (!ok) n = need = 0;
        const Pair granted = block_scan(Pair{n, need}, lds, incl);
        if (i < a.batch) {
            a.row_starts[i + 1] = (int32_t)(rows + incl.a);
            if (starts) starts[i + 1] = (int32_t)(rows + incl.a);
            if (a.granted) a.granted[i] = (int32_t)n;
            a.need[i] = (int32_t)need;
            a.at[i] = (int32_t)(pages + incl.b - need);  // counted from the first page taken, which is not known yet
        }
        rows += granted.a;
        pages += granted.b;
    }
    const int32_t left = (int32_t)(there - pages);
    for (int i = threadIdx.x; i < a.batch; i += kPageThreads) a.at[i] += left;  // the thread's own words
    if (threadIdx.x == 0) {
        a.row_starts[0] = 0;
        if (starts) starts[0] = 0;
        *a.count = left;
    }
}
__device__ __forceinline__ void release_sums(const PageArgs& a, Pair* lds) {
    const uint32_t there = min(max(*a.count, 0), a.capacity);
    uint32_t before = there;
    for (int i0 = 0; i0 < a.batch; i0 += kPageThreads) {
        const int i = i0 + threadIdx.x;
        const uint32_t n = i < a.batch ? a.need[i] : 0;
        Pair incl;
        const Pair all = block_scan(Pair{n, 0}, lds, incl);
        if (i < a.batch) a.at[i] = (int32_t)min(plus(before, incl.a) - n, (uint32_t)a.capacity);
        before = plus(before, all.a);
    }
    __syncthreads();  // every wave has read the count
    if (threadIdx.x == 0) *a.count = (int32_t)min(before, (uint32_t)a.capacity);
}

// row r; starts: row_starts, or a copy in LDS
__device__ __forceinline__ void write_row(const PageArgs& a, int64_t r, const int32_t* starts) {
    if (r >= a.max_rows) return;
    // the last request whose rows begin at or before r: those without rows begin where the next one does
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= r) lo = mid;
        else hi = mid;
    }
    const bool live = a.batch > 0 && r < starts[a.batch];
    int64_t slot = -1;
    int pos = 0;
    if (live) {
        pos = (int)(a.first[lo] + (r - starts[lo]));
        const int page = a.bt[(size_t)lo * a.width + pos / kBlockSize];
        if (page >= 0) slot = (int64_t)page * kBlockSize + pos % kBlockSize;
    }
    if (a.row_seq) a.row_seq[r] = live ? lo : -1;
    if (a.pos) a.pos[r] = pos;
    if (a.slots) a.slots[r] = slot;
}

// A grant by one workgroup.  Requests of a few columns (a token or a few more) are a thread's, the others a wave's: one column a wave
// takes as long as 512.
constexpr int kFewColumns = 4, kOneBatch = 1024;
__global__ __launch_bounds__(kPageThreads) void grant_small_kernel(PageArgs a) {
    __shared__ Pair lds[kPageWaves];
    __shared__ int many[kOneBatch], n_many, starts[kOneBatch + 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, mine = threadIdx.x;
    if (mine == 0) n_many = 0;
    __syncthreads();
    int c0 = 0, c1 = 0;
    int32_t* row = a.bt + (size_t)mine * a.width;
    if (mine < a.batch) {
        columns<true>(a, mine, c0, c1);
        if (c1 - c0 > kFewColumns) many[atomicAdd(&n_many, 1)] = mine;  // in any order: each writes its own words
        else {
            int n = 0;
#pragma unroll
            for (int u = 0; u < kFewColumns; ++u) n += c0 + u < c1 && counts<true>(row[c0 + u]);
            a.need[mine] = n;
        }
    }
    __syncthreads();
    for (int k = wave; k < n_many; k += kPageWaves) {
        const int n = count_columns<true>(a, many[k]);
        if (lane == 0) a.need[many[k]] = n;
    }
    __syncthreads();
    grant_sums(a, lds, starts);
    __syncthreads();
    if (mine < a.batch && c1 - c0 <= kFewColumns && a.need[mine] > 0) {
        int k = a.at[mine];
        for (int c = c0; c < c1; ++c)
            if (counts<true>(row[c])) move_page<true>(a, row + c, row[c], k++);
    }
    for (int k = wave; k < n_many; k += kPageWaves)
        if (a.need[many[k]] > 0) move_pages<true>(a, many[k], a.at[many[k]]);
    __syncthreads();
    if (a.row_seq || a.pos || a.slots)
        for (int64_t r = threadIdx.x; r < a.max_rows; r += kPageThreads) write_row(a, r, starts);
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
    if (GRANT) grant_sums(a, lds, nullptr);
    else release_sums(a, lds);
}
template <bool GRANT>
__global__ __launch_bounds__(256) void pages_move_kernel(PageArgs a) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i < a.batch && a.need[i] > 0) move_pages<GRANT>(a, i, a.at[i]);
}
// a workgroup's rows; where the row starts fit LDS they are searched there
constexpr int kStartsInLds = 4096;
__global__ __launch_bounds__(256) void pages_rows_kernel(PageArgs a) {
    __shared__ int32_t starts[kStartsInLds];
    const bool copied = a.batch < kStartsInLds;
    if (copied) {
        for (int i = threadIdx.x; i <= a.batch; i += 256) starts[i] = a.row_starts[i];
        __syncthreads();
    }
    write_row(a, (int64_t)blockIdx.x * 256 + threadIdx.x, copied ? starts : a.row_starts);
}

// A release of a small table in one launch: the workgroup's threads hold all of it, four entries of a row-major piece at a time, so that an
// entry's place in the list is its place in the order of the entries.
constexpr int kHeld = 8;  // pieces of four entries of a thread
__global__ __launch_bounds__(kPageThreads) void release_small_kernel(PageArgs a) {
    __shared__ Pair lds[kPageWaves];
    __shared__ int2 cols[kOneBatch];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int total = a.batch * a.width, per_wave = (total + kPageWaves * 256 - 1) / (kPageWaves * 256);  // pieces: at most kHeld
    const uint32_t there = min(max(*a.count, 0), a.capacity);
    if ((int)threadIdx.x < a.batch) {
        int c0, c1;
        columns<false>(a, threadIdx.x, c0, c1);
        cols[threadIdx.x] = make_int2(c0, c1);
    }
    int e[kHeld][4];
    const bool vec = ((uintptr_t)a.bt & 15) == 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        const int at = (wave * per_wave + k) * 256 + lane * 4;
        const bool on = k < per_wave;
        if (vec && on && at + 3 < total) {
            const int4 v = *reinterpret_cast<const int4*>(a.bt + at);
            e[k][0] = v.x, e[k][1] = v.y, e[k][2] = v.z, e[k][3] = v.w;
        } else {
#pragma unroll
            for (int z = 0; z < 4; ++z) e[k][z] = on && at + z < total ? a.bt[at + z] : -1;
        }
    }
    __syncthreads();
    uint32_t mine[kHeld], sum = 0;  // bit z: entry z goes
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        mine[k] = 0;
        const int at0 = (wave * per_wave + k) * 256, i0 = at0 / a.width, c0 = at0 - i0 * a.width;  // uniform
        if (k < per_wave && at0 < total) {
            if (c0 + 256 <= a.width) {  // the piece lies in one row
                const int2 from = cols[i0];
                const int c = c0 + lane * 4;
#pragma unroll
                for (int z = 0; z < 4; ++z) mine[k] |= (uint32_t)((e[k][z] >= 0) & (c + z >= from.x) & (c + z < from.y)) << z;
            } else {
                const int at = at0 + lane * 4;
                int i = at / a.width, c = at - i * a.width;
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    if (at + z < total) {
                        const int2 from = cols[i];
                        mine[k] |= (uint32_t)((e[k][z] >= 0) & (c >= from.x) & (c < from.y)) << z;
                    }
                    if (++c == a.width) c = 0, i = min(i + 1, a.batch - 1);
                }
            }
        }
        sum += wave_total(__popc(mine[k]));
    }
    Pair incl;
    const Pair all = block_scan(Pair{lane == 0 ? sum : 0, 0}, lds, incl);
    uint32_t place = there + (uint32_t)__builtin_amdgcn_readfirstlane((int)incl.a) - sum;  // of the wave's first
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        if (__any(mine[k] != 0)) {
            const int n = __popc(mine[k]), upto = wave_scan(n);
            uint32_t p = place + upto - n;
            const int at = (wave * per_wave + k) * 256 + lane * 4;
#pragma unroll
            for (int z = 0; z < 4; ++z)
                if (mine[k] >> z & 1) move_page<false>(a, a.bt + at + z, e[k][z], (int)p++);
            place += __builtin_amdgcn_readlane(upto, 63);
        }
    }
    __syncthreads();  // every wave has read the count
    if (threadIdx.x == 0) *a.count = (int32_t)min(there + all.a, (uint32_t)a.capacity);
}

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
    if (max_rows > 1 << 30) return fail(CHIRON_ERR_SHAPE, "pages: %d rows are too many for one call", max_rows);
    if (!out || !out->row_starts) return fail(CHIRON_ERR_INVALID_ARG, "pages: row_starts is null");
    if (!workspace || ((uintptr_t)workspace & 15)) return fail(CHIRON_ERR_INVALID_ARG, "pages: the workspace is null or not 16-byte aligned");
    if (batch > 0 && (!block_table || !seq_lens || !new_lens)) return fail(CHIRON_ERR_INVALID_ARG, "pages: a pointer argument is null");
    PageArgs a = page_args(list, block_table, max_blocks_per_seq, seq_lens, new_lens, batch, workspace);
    a.max_rows = max_rows;
    a.row_starts = out->row_starts; a.row_seq = out->row_seq; a.pos = out->pos; a.granted = out->granted; a.slots = out->slots;
    hipStream_t st = (hipStream_t)stream;
    const bool rows = out->row_seq || out->pos || out->slots;
    // One launch as far as a workgroup holds the requests and its own writing of the maps does not take longer than the other launches; us by one / by four:
    // 16 requests of 512 columns, 64 rows 10.8 / 17.2; 64 of 512, 2000 rows 11.1 / 18.1, 8000 rows 15.5 / 18.0; 1000 of 32, 1000 rows 11.4 / 19.5, 8000 15.4 / 18.6.
    if (batch <= kOneBatch && max_rows <= 8192) {
        launch(grant_small_kernel, dim3(1), dim3(kPageThreads), st, a);
    } else {
        const dim3 waves((unsigned)(((int64_t)batch + 3) / 4));
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
    // One launch as far as a workgroup's registers hold the table; us by one / by three: 16 requests of 512 columns 5.4 / 9.6, 64 of 512 7.6 / 10.3,
    // 1000 of 32 9.6 / 10.5; behind it by so little (256 of 128, every page of a full table 11.6 / 10.4) that the limit is the registers'.
    if ((int64_t)batch * max_blocks_per_seq <= kPageThreads * 4 * kHeld && batch <= kOneBatch) {
        launch(release_small_kernel, dim3(1), dim3(kPageThreads), st, a);
    } else {
        const dim3 waves((unsigned)(((int64_t)batch + 3) / 4));
        launch(pages_count_kernel<false>, waves, dim3(256), st, a);
        launch(pages_sums_kernel<false>, dim3(1), dim3(kPageThreads), st, a);
        launch(pages_move_kernel<false>, waves, dim3(256), st, a);
    }
    CHIRON_HIP(hipGetLastError());
    return CHIRON_OK;
}

}  // extern "C"
