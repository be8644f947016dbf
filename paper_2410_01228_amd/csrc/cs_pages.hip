// Whole pages of a pool, whatever is in them: copies between page lists, and what a serving loop does with a request's
// pages on the device -- forking a sequence (its full pages shared, the unfinished last one copied), freeing sequences, and
// compaction (pages in use to the front of the pool).  Page counts, tables and lists stay on the device: no call waits for one.
#include <algorithm>
#include "cs_common.h"

namespace cs {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------
// Copies: HBM-bound, 16 bytes a lane past the caches, a wavefront a KiB as in the checkpoint copies (many small workgroups
// sustain more bandwidth on this part than fewer, fatter ones).  Workgroups are dealt round-robin to the 8 XCDs, each with its
// own L2 and address translation; here all chunks of a page go to one of them: 1152 pages of 32832 bytes, 48 layers, between
// shuffled places 4.87 -> 5.47 TB/s (read + write), 576 of 65536 6.09 -> 6.19, 3100 of 16416 (28 layers) 5.15 -> 5.35.  Chunks of 2 to
// 16 KiB a workgroup of 64 to 1024 threads are within 2% of that or slower, layers side by side up to 8% slower; what is left
// to the 6.79 TB/s of a contiguous copy are the shuffled pages.
// ------------------------------------------------------------------------------------
constexpr int kLanes = 64, kXcds = 8;

inline int32_t chunks_of(int64_t page_bytes, int64_t chunk) { return (int32_t)std::max<int64_t>(1, page_bytes / chunk); }

// The page and chunk of workgroup x of a grid of `padded(pages) * chunks`.
inline int64_t padded(int64_t pages) { return (pages + kXcds - 1) / kXcds * kXcds; }
__device__ __forceinline__ void deal(uint32_t x, int32_t chunks, int32_t& page, int32_t& chunk) {
    const uint32_t k = x / kXcds, j = k / (uint32_t)chunks;
    page = (int32_t)(j * kXcds + (x & (kXcds - 1)));
    chunk = (int32_t)(k - j * (uint32_t)chunks);
}

// Chunk c of a page, U runs of 16 bytes a lane: the last one takes what is left behind the last whole chunk along (the scales of
// an 8-bit page are 64 bytes behind 32 KiB).
template <int T, int U = 1, bool kReadAgain = false>
__device__ __forceinline__ void copy_chunk(char* dst, const char* src, int32_t c, int32_t chunks, int64_t bytes) {
    constexpr int kRun = T * 16;
    const int64_t begin = (int64_t)c * (kRun * U) + threadIdx.x * 16, end = c == chunks - 1 ? bytes : begin + kRun * U;
    for (int64_t off = begin; off < end; off += kRun * (U + 1)) {
        u32x4 r[U + 1];                                           // (one more: what is left over is less than a chunk)
#pragma unroll
        for (int u = 0; u <= U; ++u)
            if (off + u * kRun < end) {
                const u32x4* p = (const u32x4*)(src + off + u * kRun);
                r[u] = kReadAgain ? *p : __builtin_nontemporal_load(p);
            }
#pragma unroll
        for (int u = 0; u <= U; ++u)
            if (off + u * kRun < end) __builtin_nontemporal_store(r[u], (u32x4*)(dst + off + u * kRun));
    }
}

// A pool as the kernels see it.
struct Pages {
    char* base;
    int64_t layer_stride, page_stride;
    int32_t num_pages;
    __device__ __forceinline__ bool has(int32_t id) const { return id >= 0 && id < num_pages; }
    __device__ __forceinline__ char* at(int32_t layer, int32_t id) const { return base + (int64_t)layer * layer_stride + (int64_t)id * page_stride; }
};

// grid = (padded(pages) * chunks_per_page, layers); pages first .. first + n - 1 of the lists; ids: null for 0, 1, 2, ...
__global__ __launch_bounds__(kLanes) void pages_copy_kernel(const Pages src, const int32_t* __restrict__ src_ids, const Pages dst,
                                                            const int32_t* __restrict__ dst_ids, int32_t first, int32_t n, int64_t page_bytes, int32_t chunks_per_page)
{
    int32_t k, c;
    deal(blockIdx.x, chunks_per_page, k, c);
    if (k >= n) return;
    const int32_t i = first + k;
    const int32_t from = src_ids ? src_ids[i] : i, to = dst_ids ? dst_ids[i] : i;
    if (!src.has(from) || !dst.has(to)) return;
    copy_chunk<kLanes>(dst.at(blockIdx.y, to), src.at(blockIdx.y, from), c, chunks_per_page, page_bytes);
}

// ------------------------------------------------------------------------------------
// Forks and frees
// ------------------------------------------------------------------------------------
struct Tables {
    int32_t* entries;
    int32_t* lens;
    int32_t* counts;
    int32_t num_rows, max_blocks, num_pages, page_size;
    __device__ __forceinline__ bool has_row(int32_t r) const { return r >= 0 && r < num_rows; }
    __device__ __forceinline__ bool has_page(int32_t id) const { return id >= 0 && id < num_pages; }
    // tokens of a row, at most what its entries hold
    __device__ __forceinline__ int32_t tokens(int32_t n) const { return (int32_t)min((int64_t)max(n, 0), (int64_t)max_blocks * page_size); }
};

// grid = (padded(forks) * chunks_per_page, layers + 1).  Planes 0 .. layers - 1 copy the unfinished last pages, a chunk a workgroup;
// the last plane writes the children's rows and counts, the workgroups of a fork 64 entries each in turn.  Neither
// reads what the other writes: a child is no parent.  A chunk is 4 KiB here: three loads in a row say where it is.
constexpr int kForkRuns = 4;
__global__ __launch_bounds__(kLanes) void pages_fork_kernel(const Pages pool, int64_t page_bytes, int32_t chunks_per_page, int32_t layers, const Tables t,
                                                            const int32_t* __restrict__ parents, const int32_t* __restrict__ children,
                                                            const int32_t* __restrict__ fresh_pages, int32_t n_forks)
{
    // neighbours in the list on one XCD: they often have the same parent, whose page then comes from its L2 (64 parents, 8 children each,
    // 80 layers of 32832 bytes: 489 -> 252 us)
    int32_t i, c;
    deal(blockIdx.x, chunks_per_page, i, c);
    i = (i & (kXcds - 1)) * (int32_t)(gridDim.x / ((uint32_t)chunks_per_page * kXcds)) + i / kXcds;
    if (i >= n_forks) return;
    const int32_t parent = parents[i], child = children[i], fresh = fresh_pages[i];
    if (!t.has_row(parent) || !t.has_row(child)) return;
    int32_t n = t.tokens(t.lens[parent]);
    const int32_t full = n / t.page_size;
    const bool tail = n > full * t.page_size;
    const int32_t* from = t.entries + (int64_t)parent * t.max_blocks;
    const int32_t last = tail ? from[full] : -1;
    const bool copied = pool.has(last) && pool.has(fresh);
    if ((int32_t)blockIdx.y < layers) {
        if (copied) copy_chunk<kLanes, kForkRuns, true>(pool.at(blockIdx.y, fresh), pool.at(blockIdx.y, last), c, chunks_per_page, page_bytes);
        return;
    }
    if (!copied) n = full * t.page_size;                          // no page for the rest, or no rest: the child ends at its last full one
    int32_t* to = t.entries + (int64_t)child * t.max_blocks;
    for (int32_t e = c * kLanes + threadIdx.x; e < t.max_blocks; e += chunks_per_page * kLanes) {
        int32_t id = -1;
        if (e < full) {
            id = from[e];
            if (t.has_page(id)) atomicAdd(t.counts + id, 1);
        } else if (e == full && copied) {
            id = fresh;
            t.counts[id] = 1;
        }
        to[e] = id;
    }
    if (c == 0 && threadIdx.x == 0) t.lens[child] = n;
}

// Counts that reach zero in a call are marked until the list is written: far below zero, so that a page given back
// more often than it was held (a mistake of the caller's, undone on the spot) cannot pass for one.
constexpr int32_t kFreed = 1 << 30;

constexpr int kFreeThreads = 256;
__global__ __launch_bounds__(kFreeThreads) void pages_release_kernel(const Tables t, const int32_t* __restrict__ rows)
{
    const int32_t r = rows[blockIdx.x];
    if (!t.has_row(r)) return;
    __shared__ int32_t len;
    if (threadIdx.x == 0) len = atomicExch(t.lens + r, 0);        // a row listed twice is freed once
    __syncthreads();
    const int32_t n = (int32_t)(((int64_t)t.tokens(len) + t.page_size - 1) / t.page_size);
    int32_t* row = t.entries + (int64_t)r * t.max_blocks;
    for (int32_t e = threadIdx.x; e < n; e += kFreeThreads) {
        const int32_t id = row[e];
        row[e] = -1;
        if (!t.has_page(id)) continue;
        const int32_t before = atomicSub(t.counts + id, 1);
        if (before == 1) atomicSub(t.counts + id, kFreed);
        else if (before <= 0) atomicAdd(t.counts + id, 1);
    }
}

// One workgroup walks over all pages in order, kPer of them a lane and trip: wavefront w of a trip has kPer * 64 consecutive
// ones, row after row of 64, so that loads and stores are whole lines and a page's rank among the listed ones comes from
// ballots.  The order of a list is the pages' own, whatever the wavefronts do.  Bound by latency: the next trip's counts are on
// their way during this one.
constexpr int kScanThreads = 1024, kScanWaves = kScanThreads / 64, kPer = 8, kTrip = kScanThreads * kPer;
struct ScanLds { int32_t sum[2][kScanWaves]; };                   // (two: a trip writes the one that the trip before last read)

__device__ __forceinline__ int64_t page_of(int64_t base, int j) { return base + (threadIdx.x >> 6) * (kPer * 64) + j * 64 + (threadIdx.x & 63); }
__device__ __forceinline__ void load_counts(int32_t (&c)[kPer], const int32_t* counts, int64_t base, int32_t n)
{
#pragma unroll
    for (int j = 0; j < kPer; ++j) c[j] = page_of(base, j) < n ? counts[page_of(base, j)] : 0;
}
// Lanes below this one in a ballot.
__device__ __forceinline__ int32_t below(uint64_t ballot) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(ballot >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)ballot, 0)); }
// The sum of `mine`, a wavefront's own, over the wavefronts before this one; total: over all of them.
__device__ __forceinline__ int32_t sum_before(int32_t mine, int trip, ScanLds& lds, int32_t& total)
{
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds.sum[trip & 1][wave] = mine;
    __syncthreads();
    int32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kScanWaves; ++w) {
        const int32_t v = lds.sum[trip & 1][w];
        if (w < wave) before += v;
        total += v;
    }
    return before;
}

__global__ __launch_bounds__(kScanThreads) void pages_freed_kernel(int32_t* __restrict__ counts, int32_t num_pages, int32_t* __restrict__ freed,
                                                                   int32_t* __restrict__ num_freed)
{
    __shared__ ScanLds lds;
    int32_t listed = 0, c[kPer], next[kPer];
    load_counts(c, counts, 0, num_pages);
    int trip = 0;
    for (int64_t base = 0; base < num_pages; base += kTrip, ++trip) {
        load_counts(next, counts, base + kTrip, num_pages);
        uint64_t hit[kPer];
        int32_t mine = 0, total;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            hit[j] = __ballot(c[j] <= -(kFreed / 2));
            mine += __popcll(hit[j]);
        }
        int32_t rank = listed + sum_before(mine, trip, lds, total);
        listed += total;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (c[j] <= -(kFreed / 2)) {
                freed[rank + below(hit[j])] = (int32_t)page_of(base, j);
                counts[page_of(base, j)] = 0;
            }
            rank += __popcll(hit[j]);
            c[j] = next[j];
        }
    }
    if (threadIdx.x == 0) *num_freed = listed;
}

// ------------------------------------------------------------------------------------
// Compaction: with n pages in use, the k-th used page from n on moves to the k-th free page below n.
// ------------------------------------------------------------------------------------
// Workspace: this, then for each move to[], from[] and the count that moves, most_moves() of each.
struct Moves { int32_t n, pad[3]; };
__host__ __device__ inline int64_t most_moves(int32_t num_pages) { return num_pages / 2 + 1; }

__global__ __launch_bounds__(kScanThreads) void pages_plan_kernel(const int32_t* counts, int32_t num_pages, int32_t* new_counts,
                                                                  int32_t* __restrict__ new_ids, int32_t* __restrict__ num_used, Moves* __restrict__ moves)
{
    __shared__ ScanLds lds;
    int32_t* to = (int32_t*)(moves + 1);
    int32_t* from = to + most_moves(num_pages);
    int32_t* held = from + most_moves(num_pages);
    int32_t used = 0, c[kPer], next[kPer];
    {
        int32_t mine = 0;
        load_counts(c, counts, 0, num_pages);
        for (int64_t base = 0; base < num_pages; base += kTrip) {
            load_counts(next, counts, base + kTrip, num_pages);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                mine += __popcll(__ballot(c[j] > 0));
                c[j] = next[j];
            }
        }
        load_counts(c, counts, 0, num_pages);
        sum_before(mine, 1, lds, used);
    }
    int32_t holes = 0, movers = 0;
    int trip = 0;
    for (int64_t base = 0; base < num_pages; base += kTrip, ++trip) {
        load_counts(next, counts, base + kTrip, num_pages);
        // (below `used` holes are counted, from it on movers: both in one sum, 16 bits each, of at most 8192 a trip)
        uint64_t hole[kPer], mover[kPer];
        int32_t mine = 0, total;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int64_t p = page_of(base, j);
            hole[j] = __ballot(p < used && c[j] <= 0);
            mover[j] = __ballot(p >= used && c[j] > 0);          // (no page behind the last one has a count)
            mine += __popcll(hole[j]) + (__popcll(mover[j]) << 16);
        }
        const int32_t before = sum_before(mine, trip, lds, total);
        int32_t h = holes + (before & 0xffff), m = movers + (before >> 16);
        holes += total & 0xffff;
        movers += total >> 16;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int64_t p = page_of(base, j);
            if (p < used && c[j] <= 0) {
                to[h + below(hole[j])] = (int32_t)p;
            } else if (p >= used && c[j] > 0) {
                from[m + below(mover[j])] = (int32_t)p;
                held[m + below(mover[j])] = c[j];
            } else if (p < num_pages) {
                new_ids[p] = c[j] > 0 ? (int32_t)p : -1;
                new_counts[p] = c[j] > 0 ? c[j] : 0;
            }
            h += __popcll(hole[j]);
            m += __popcll(mover[j]);
            c[j] = next[j];
        }
    }
    __threadfence_block();
    __syncthreads();
    // (as many of the one as of the other)
    constexpr int kAtOnce = 4;
    for (int32_t k0 = threadIdx.x; k0 < movers; k0 += kScanThreads * kAtOnce) {
        int32_t a[kAtOnce], b[kAtOnce], n[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int32_t k = min(k0 + j * kScanThreads, movers - 1);
            a[j] = from[k];
            b[j] = to[k];
            n[j] = held[k];
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (k0 + j * kScanThreads >= movers) break;
            new_ids[a[j]] = b[j];
            new_ids[b[j]] = -1;
            new_counts[b[j]] = n[j];
            new_counts[a[j]] = 0;
        }
    }
    if (threadIdx.x == 0) {
        moves->n = movers;
        *num_used = used;
    }
}

// The first table_wgs workgroups (a multiple of the XCDs) renumber the tables; the others copy the moved pages, every eighth of
// them by the workgroups of one XCD, chunk by chunk in turn, as many as the planning kernel found (the host does not know).
// 64 workgroups a CU, of which four are resident: 3100 pages of 16416 bytes, 28 layers, 5.37 TB/s; 5.21 with 32, 4.84 with 8, 4.16
// with two, the same with as many lanes in workgroups of 64 or 256.
constexpr int kWide = 512, kApplyPerCu = 64;
__global__ __launch_bounds__(kWide) void pages_apply_kernel(const Pages pool, int64_t page_bytes, int32_t chunks_per_page, int32_t layers,
                                                            const Tables t, int32_t* new_entries, const int32_t* __restrict__ new_ids,
                                                            const Moves* __restrict__ moves, uint32_t table_wgs)
{
    if (blockIdx.x < table_wgs) {
        const int64_t n = (int64_t)t.num_rows * t.max_blocks;
        for (int64_t e = (int64_t)blockIdx.x * kWide + threadIdx.x; e < n; e += (int64_t)table_wgs * kWide) {
            const int32_t row = (int32_t)(e / t.max_blocks), b = (int32_t)(e - (int64_t)row * t.max_blocks);
            int32_t id = -1;
            if ((int64_t)b * t.page_size < t.tokens(t.lens[row])) {
                id = t.entries[e];
                id = t.has_page(id) ? new_ids[id] : -1;
            }
            new_entries[e] = id;
        }
        return;
    }
    const int32_t* to = (const int32_t*)(moves + 1);
    const int32_t* from = to + most_moves(t.num_pages);
    const int32_t xcd = blockIdx.x % kXcds, n = (moves->n - xcd + kXcds - 1) / kXcds;     // moves of this XCD
    const int64_t per_layer = (int64_t)n * chunks_per_page, total = per_layer * layers, wgs = (gridDim.x - table_wgs) / kXcds;
    for (int64_t w = (blockIdx.x - table_wgs) / kXcds; w < total; w += wgs) {
        const int32_t l = (int32_t)(w / per_layer);
        const int64_t rem = w - l * per_layer;
        const int32_t j = (int32_t)(rem / chunks_per_page), c = (int32_t)(rem - (int64_t)j * chunks_per_page), k = j * kXcds + xcd;
        copy_chunk<kWide>(pool.at(l, to[k]), pool.at(l, from[k]), c, chunks_per_page, page_bytes);
    }
}

static int validate_space(const cs_page_space* s) {
    if (!s || !s->base || ((uintptr_t)s->base & 15)) return CS_ERR_INVALID_ARG;
    if (s->num_layers <= 0 || s->num_pages <= 0 || s->page_bytes <= 0) return CS_ERR_INVALID_ARG;
    if ((s->page_bytes & 15) || (s->page_stride & 15) || (s->layer_stride & 15)) return CS_ERR_INVALID_ARG;
    if (s->page_bytes > (1ll << 30)) return CS_ERR_UNSUPPORTED;
    if (s->page_stride < s->page_bytes || s->page_stride > INT64_MAX / s->num_pages) return CS_ERR_INVALID_ARG;
    return s->layer_stride < s->page_stride * s->num_pages && s->num_layers > 1 ? CS_ERR_INVALID_ARG : CS_OK;
}

static int validate_tables(const cs_page_tables* t) {
    if (!t || !t->block_tables || !t->lens || !t->ref_counts) return CS_ERR_INVALID_ARG;
    if (t->num_rows <= 0 || t->max_blocks_per_seq <= 0 || t->num_pages <= 0 || t->page_size <= 0) return CS_ERR_INVALID_ARG;
    return CS_OK;
}

static bool layers_ok(const cs_page_space& s, int32_t l0, int32_t l1) { return l0 >= 0 && l1 >= l0 && l1 <= s.num_layers && l1 - l0 < 65535; }
static Pages pages_of(const cs_page_space& s, int32_t layer) {
    return Pages{(char*)s.base + (int64_t)layer * s.layer_stride, s.layer_stride, s.page_stride, s.num_pages};
}
static Tables tables_of(const cs_page_tables& t) {
    return Tables{t.block_tables, t.lens, t.ref_counts, t.num_rows, t.max_blocks_per_seq, t.num_pages, t.page_size};
}

constexpr int64_t kMostLanes = 4294967295ll;                      // of a launch, along x

}  // namespace cs

using namespace cs;

extern "C" {

int cs_kv_page_space(const cs_kv_pool* pool, cs_page_space* space) {
    const int rc = validate_pool(pool);
    if (rc) return rc;
    if (!space) return CS_ERR_INVALID_ARG;
    *space = cs_page_space{pool->base, pool->num_layers, pool->num_pages, (int64_t)pool_page_bytes(*pool), pool->layer_stride * 2, pool->page_stride * 2};
    return CS_OK;
}

int cs_kv_pages_copy(const cs_page_space* src, int32_t src_layer, const int32_t* src_ids, const cs_page_space* dst, int32_t dst_layer,
                     const int32_t* dst_ids, int32_t num_layers, int32_t n, void* stream) {
    int rc = validate_space(src);
    if (rc == CS_OK) rc = validate_space(dst);
    if (rc) return rc;
    if (num_layers < 0 || n < 0 || src->page_bytes != dst->page_bytes) return CS_ERR_INVALID_ARG;
    if (src_layer < 0 || src_layer > src->num_layers || num_layers > src->num_layers - src_layer) return CS_ERR_INVALID_ARG;
    if (dst_layer < 0 || dst_layer > dst->num_layers || num_layers > dst->num_layers - dst_layer || num_layers > 65535) return CS_ERR_INVALID_ARG;
    if ((!src_ids && n > src->num_pages) || (!dst_ids && n > dst->num_pages)) return CS_ERR_INVALID_ARG;
    if (n == 0 || num_layers == 0) return CS_OK;
    const int32_t cpp = chunks_of(src->page_bytes, kLanes * 16);
    const int32_t most = (int32_t)std::max<int64_t>(kXcds, std::min<int64_t>(n, kMostLanes / kLanes / cpp / kXcds * kXcds));
    for (int32_t first = 0; first < n; first += std::min(most, n - first)) {
        const int32_t m = std::min(most, n - first);
        hipLaunchKernelGGL(pages_copy_kernel, dim3((uint32_t)(padded(m) * cpp), (uint32_t)num_layers), dim3(kLanes), 0, (hipStream_t)stream,
                           pages_of(*src, src_layer), src_ids, pages_of(*dst, dst_layer), dst_ids, first, m, src->page_bytes, cpp);
    }
    return check_launch("page copy kernel");
}

int cs_kv_pages_fork(const cs_page_space* space, int32_t layer_begin, int32_t layer_end, const cs_page_tables* tables, const int32_t* parents,
                     const int32_t* children, const int32_t* fresh_pages, int32_t n, void* stream) {
    int rc = validate_space(space);
    if (rc == CS_OK) rc = validate_tables(tables);
    if (rc) return rc;
    if (!layers_ok(*space, layer_begin, layer_end) || n < 0 || tables->num_pages != space->num_pages) return CS_ERR_INVALID_ARG;
    if (n == 0) return CS_OK;
    if (!parents || !children || !fresh_pages) return CS_ERR_INVALID_ARG;
    const int32_t cpp = chunks_of(space->page_bytes, kLanes * 16 * kForkRuns), layers = layer_end - layer_begin;
    if (padded(n) * cpp * kLanes > kMostLanes) return CS_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(pages_fork_kernel, dim3((uint32_t)(padded(n) * cpp), (uint32_t)layers + 1), dim3(kLanes), 0, (hipStream_t)stream,
                       pages_of(*space, layer_begin), space->page_bytes, cpp, layers, tables_of(*tables), parents, children, fresh_pages, n);
    return check_launch("page fork kernel");
}

int cs_kv_pages_free(const cs_page_tables* tables, const int32_t* rows, int32_t n, int32_t* freed, int32_t* num_freed, void* stream) {
    const int rc = validate_tables(tables);
    if (rc) return rc;
    if (n < 0 || !freed || !num_freed || (n > 0 && !rows)) return CS_ERR_INVALID_ARG;
    if ((int64_t)n * kFreeThreads > kMostLanes) return CS_ERR_UNSUPPORTED;
    if (n > 0) hipLaunchKernelGGL(pages_release_kernel, dim3((uint32_t)n), dim3(kFreeThreads), 0, (hipStream_t)stream, tables_of(*tables), rows);
    hipLaunchKernelGGL(pages_freed_kernel, dim3(1), dim3(kScanThreads), 0, (hipStream_t)stream, tables->ref_counts, tables->num_pages, freed, num_freed);
    return check_launch("page free kernels");
}

size_t cs_kv_pages_compact_workspace_bytes(int32_t num_pages) {
    return num_pages <= 0 ? 0 : sizeof(Moves) + 3 * (size_t)most_moves(num_pages) * sizeof(int32_t);
}

int cs_kv_pages_compact(const cs_page_space* space, int32_t layer_begin, int32_t layer_end, const cs_page_tables* tables, const cs_page_tables* new_tables,
                        int32_t* new_ids, int32_t* num_used, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = validate_space(space);
    if (rc == CS_OK) rc = validate_tables(tables);
    if (rc == CS_OK) rc = validate_tables(new_tables);
    if (rc) return rc;
    if (!layers_ok(*space, layer_begin, layer_end) || tables->num_pages != space->num_pages || new_tables->num_pages != space->num_pages ||
        new_tables->num_rows != tables->num_rows || new_tables->max_blocks_per_seq != tables->max_blocks_per_seq || new_tables->page_size != tables->page_size)
        return CS_ERR_INVALID_ARG;
    if (!new_ids || !num_used || !workspace || ((uintptr_t)workspace & 15)) return CS_ERR_INVALID_ARG;
    if (workspace_bytes < cs_kv_pages_compact_workspace_bytes(space->num_pages)) return CS_ERR_WORKSPACE_TOO_SMALL;
    hipStream_t st = (hipStream_t)stream;
    Moves* moves = (Moves*)workspace;
    hipLaunchKernelGGL(pages_plan_kernel, dim3(1), dim3(kScanThreads), 0, st, tables->ref_counts, space->num_pages, new_tables->ref_counts, new_ids, num_used, moves);
    const int64_t entries = (int64_t)tables->num_rows * tables->max_blocks_per_seq;
    const uint32_t table_wgs = (uint32_t)padded(std::min<int64_t>((entries + kWide - 1) / kWide, device_cus()));
    const int32_t layers = layer_end - layer_begin, cpp = chunks_of(space->page_bytes, kWide * 16);
    const uint32_t copy_wgs = (uint32_t)padded(std::min<int64_t>(most_moves(space->num_pages) * layers * cpp, (int64_t)kApplyPerCu * device_cus()));
    hipLaunchKernelGGL(pages_apply_kernel, dim3(table_wgs + copy_wgs), dim3(kWide), 0, st, pages_of(*space, layer_begin), space->page_bytes, cpp, layers,
                       tables_of(*tables), new_tables->block_tables, new_ids, moves, table_wgs);
    return check_launch("page compaction kernels");
}

}  // extern "C"
