// The paged cache of a serving node: the bookkeeping of a step (fedrag_paged_map) and its rows' way into the pages
// (fedrag_paged_write).
#include "fedrag_device.h"
#include "fedrag_host.h"

#include <climits>

namespace fedrag {

// ------------------------------------------------------------------------------------------------ map
// One workgroup takes the requests 1024 at a time: prefix sums of their rows (which end at n_rows: min(a + b, n_rows) is
// associative as + is) and of the pages they take, carried from one thousand to the next.  Each new page is then a thread's,
// which finds its request in the prefix sums, and so is each row, up to kMapRows of them; beyond, the rows are a launch of
// their own over the whole chip, which reads what this one has written.  Bound by the chain of its steps: a launch that reads
// and writes a few KB (4.8 us for 4 decoding requests, 7.0 for 256 with some chunks of prompts; 32 prompts of 4000 tokens 8.3 and 3.6).
// A thread reads a request's lengths before it writes them, and the second launch takes what the first has written: that is what lets
// a step advance in place.
constexpr int kMapThreads = 1024;

struct MapPrefix {
    uint32_t rows, pages;
};
// Inclusive prefix sums over the workgroup; total: those of all threads.
__device__ __forceinline__ MapPrefix map_scan(MapPrefix x, uint32_t most_rows, MapPrefix (&waves)[kMapThreads / kWave], MapPrefix* total) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t r = __shfl_up(x.rows, o), p = __shfl_up(x.pages, o);
        if (lane >= o) {
            x.rows = min(x.rows + r, most_rows);
            x.pages += p;
        }
    }
    if (lane == kWave - 1) waves[wave] = x;
    __syncthreads();
    MapPrefix before{0, 0}, all{0, 0};
#pragma unroll
    for (int w = 0; w < kMapThreads / kWave; ++w) {
        if (w == wave) before = all;
        all.rows = min(all.rows + waves[w].rows, most_rows);
        all.pages += waves[w].pages;
    }
    *total = all;
    return MapPrefix{min(before.rows + x.rows, most_rows), before.pages + x.pages};
}
// The first of n nondecreasing numbers that is above x.
__device__ __forceinline__ int first_above(const uint32_t* v, int n, uint32_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (v[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

FEDRAG_KERNEL __launch_bounds__(kMapThreads) void paged_map_kernel(PagedMapJob j, int shift, int rows_too) {
    __shared__ MapPrefix waves[kMapThreads / kWave];
    __shared__ uint32_t row_end[kMapThreads], page_end[kMapThreads];
    __shared__ int cached[kMapThreads], had_pages[kMapThreads];
    __shared__ int flags;
    const int tid = threadIdx.x;
    const uint32_t n_rows = (uint32_t)j.n_rows;
    const int64_t max_pages = j.max_pages;
    const int count_in = *j.free_count;
    const int64_t count = count_in < 0 ? 0 : (count_in < j.n_free ? count_in : j.n_free);
    if (tid == 0) flags = count_in == count ? 0 : FEDRAG_MAP_BAD_LENGTH;
    uint32_t rows0 = 0, pages0 = 0;  // of the requests before this thousand
    for (int64_t b0 = 0; b0 < j.batch; b0 += kMapThreads) {
        __syncthreads();
        const int64_t b = b0 + tid;
        const int n_req = (int)(j.batch - b0 < kMapThreads ? j.batch - b0 : kMapThreads);
        int c = 0, n = 0, mine = 0;
        if (b < j.batch) {
            c = j.cached_lens[b];
            n = j.new_lens[b];
            if (c < 0 || n < 0) mine |= FEDRAG_MAP_BAD_LENGTH;
            c = c < 0 ? 0 : c;
            n = n < 0 ? 0 : n;
            if ((uint32_t)n > n_rows) {
                n = (int)n_rows;
                mine |= FEDRAG_MAP_NO_ROWS;
            }
            if (c > INT_MAX - n) {
                c = INT_MAX - n;
                mine |= FEDRAG_MAP_BAD_LENGTH;
            }
        }
        // rows first: they decide how many of the new tokens there are
        MapPrefix total;
        const MapPrefix r = map_scan(MapPrefix{(uint32_t)n, 0}, n_rows, waves, &total);
        const uint32_t end = min(rows0 + r.rows, n_rows);
        const uint32_t rows1 = min(rows0 + total.rows, n_rows);
        row_end[tid] = end;
        __syncthreads();
        const uint32_t start = tid == 0 ? rows0 : row_end[tid - 1];
        if ((int)(end - start) < n) mine |= FEDRAG_MAP_NO_ROWS;
        n = (int)(end - start);
        const int64_t need = ((int64_t)c + n + (1 << shift) - 1) >> shift;
        int64_t had = ((int64_t)c + (1 << shift) - 1) >> shift;
        if (need > max_pages) mine |= FEDRAG_MAP_NO_COLUMNS;
        had = had < max_pages ? had : max_pages;
        const int64_t want = (need < max_pages ? need : max_pages) - had;
        const MapPrefix p = map_scan(MapPrefix{0, (uint32_t)(want > 0 ? want : 0)}, n_rows, waves, &total);
        const uint32_t pages1 = pages0 + total.pages;
        if (pages0 + p.pages > count && want > 0) mine |= FEDRAG_MAP_NO_PAGES;
        page_end[tid] = pages0 + p.pages;
        cached[tid] = c;
        had_pages[tid] = (int)had;
        if (b < j.batch) {
            j.q_start[b] = (int)start;
            j.kv_lens[b] = c + n;
        }
        if (mine) atomicOr(&flags, mine);
        __syncthreads();
        auto fresh = [&](uint32_t i) { return i < count ? j.free_pages[count - 1 - i] : -1; };
        for (uint32_t i = pages0 + tid; i < pages1; i += kMapThreads) {
            const int k = first_above(page_end, n_req, i);
            const uint32_t first = k == 0 ? pages0 : page_end[k - 1];
            j.block_table[(b0 + k) * max_pages + had_pages[k] + (i - first)] = fresh(i);
        }
        if (rows_too)
            for (uint32_t t = rows0 + tid; t < rows1; t += kMapThreads) {
                const int k = first_above(row_end, n_req, t);
                const int pos = cached[k] + (int)(t - (k == 0 ? rows0 : row_end[k - 1]));
                const int col = pos >> shift;
                const uint32_t first = k == 0 ? pages0 : page_end[k - 1];
                int id = -1;
                if (col < max_pages)
                    id = col < had_pages[k] ? j.block_table[(b0 + k) * max_pages + col] : fresh(first + (uint32_t)(col - had_pages[k]));
                j.slots[t] = id < 0 ? -1 : ((int64_t)id << shift) + (pos & ((1 << shift) - 1));
                if (j.positions) j.positions[t] = pos;
            }
        rows0 = rows1;
        pages0 = pages1;
    }
    if (rows_too)
        for (uint32_t t = rows0 + tid; t < n_rows; t += kMapThreads) {
            j.slots[t] = -1;
            if (j.positions) j.positions[t] = -1;
        }
    __syncthreads();
    if (tid == 0) {
        j.q_start[j.batch] = (int)rows0;
        *j.free_left = (int)(count - (pages0 < count ? pages0 : count));
        *j.flags = flags;
    }
}

// The rows of a step whose requests are planned.  A wave looks for its first row's and its last row's request, 64 candidates a
// trip to memory; mostly the two are one.
__device__ __forceinline__ int request_of(const int32_t* q_start, int batch, int t) {
    int lo = 0, n = batch;  // the request is the last whose start is <= t among lo .. lo + n - 1
    const int lane = threadIdx.x % kWave;
    while (n > 1) {
        const int step = (n + kWave - 1) / kWave;
        const int i = lane * step;
        const int s = i < n ? q_start[lo + i] : INT_MAX;
        const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(s <= t)) - 1;  // starts do not decrease
        const int at = k < 0 ? 0 : k * step;
        lo += at;
        n = n - at < step ? n - at : step;
    }
    return lo;
}
FEDRAG_KERNEL __launch_bounds__(256) void paged_map_rows_kernel(PagedMapJob j, int shift) {
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x / kWave * kWave, t = first + threadIdx.x % kWave;
    if (first >= j.n_rows) return;
    const int rows = j.batch > 0 ? j.q_start[j.batch] : 0;
    int64_t slot = -1;
    int pos = -1;
    if (first < rows) {
        const int last = (int)(first + kWave < rows ? first + kWave : rows) - 1;
        int lo = __builtin_amdgcn_readfirstlane(request_of(j.q_start, j.batch, (int)first)), hi = lo;
        if (last >= j.q_start[lo + 1]) hi = __builtin_amdgcn_readfirstlane(request_of(j.q_start, j.batch, last));
        if (t < rows) {
            while (lo < hi) {  // the last request that starts at or before t
                const int mid = hi - (hi - lo) / 2;
                if (j.q_start[mid] <= t) lo = mid;
                else hi = mid - 1;
            }
            pos = j.kv_lens[lo] - j.q_start[lo + 1] + (int)t;
            const int col = pos >> shift;
            const int id = col < j.max_pages ? j.block_table[lo * j.max_pages + col] : -1;
            if (id >= 0) slot = ((int64_t)id << shift) + (pos & ((1 << shift) - 1));
        }
    }
    if (t >= j.n_rows) return;
    j.slots[t] = slot;
    if (j.positions) j.positions[t] = pos;
}

// Rows that the one workgroup maps itself: a launch less, but a chip less too (one launch and two: 4 requests of 1000 rows 6.3 and
// 7.5 us, 1 of 4096 6.1 and 6.9, 8 of 1000 8.8 and 7.6, 256 of 32 11.2 and 8.3, 32 of 1000 26 and 8.5).
constexpr int64_t kMapRows = 4096;

hipError_t launch_paged_map(const PagedMapJob& job, hipStream_t stream) {
    const int shift = __builtin_ctz((unsigned)job.page_tokens);
    const int rows_too = job.n_rows <= kMapRows ? 1 : 0;
    hipLaunchKernelGGL(paged_map_kernel, dim3(1), dim3(kMapThreads), 0, stream, job, shift, rows_too);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || rows_too) return e;
    hipLaunchKernelGGL(paged_map_rows_kernel, dim3((unsigned)((job.n_rows + 255) / 256)), dim3(256), 0, stream, job, shift);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ write
// A copy: a thread moves 16 bytes of one row of one head, K's or V's.  A workgroup takes rows that follow each other in the
// step, whose places in a page mostly follow each other too: whole runs of a page are written at once, and of a projection's
// output whole rows of a head are read.  Bound by HBM: 32768 rows of 8 heads of 128 48.4 us, 5.55 TB/s of bytes read and written (a
// library copy of 1 GiB 5.1); a single row 2.5 us, most of it the slot's trip and then the row's.
constexpr int kWriteThreads = 256;

template <int CH>  // 16-byte chunks per row
FEDRAG_KERNEL __launch_bounds__(kWriteThreads) void paged_write_kernel(PagedWriteJob j) {
    constexpr int kRows = kWriteThreads / CH;
    const int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / CH;
    const int c = threadIdx.x % CH * 16;
    const int h = blockIdx.y, which = blockIdx.z;
    if (t >= j.n_rows) return;
    const int64_t slot = j.slots[t];
    if (slot < 0 || slot >= ((int64_t)j.pages.n_pages << j.pages.shift)) return;
    const char* from = (const char*)j.rows[which] + h * j.head_stride[which] + t * j.token_stride[which] + c;
    char* to = (char*)(which ? j.pages.V : j.pages.K) + (slot >> j.pages.shift) * j.pages.page_bytes +
               (((int64_t)h << j.pages.shift) + (slot & ((1 << j.pages.shift) - 1))) * (CH * 16) + c;
    *(u32x4_t*)to = *(const u32x4_t*)from;
}

static int64_t write_groups(const PagedWriteJob& job) {  // workgroups for the rows of a head
    const int64_t rows = kWriteThreads / (job.D * job.elem_bytes / 16);
    return (job.n_rows + rows - 1) / rows;
}
bool paged_write_fits(const PagedWriteJob& job) { return job.H <= 65535 && grid_fits(write_groups(job) * job.H * 2, kWriteThreads); }

hipError_t launch_paged_write(const PagedWriteJob& job, hipStream_t stream) {
    const int chunks = job.D * job.elem_bytes / 16;
    const int64_t groups = write_groups(job);
    const auto kernel = chunks == 8 ? paged_write_kernel<8> : chunks == 16 ? paged_write_kernel<16> : paged_write_kernel<32>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)job.H, 2), dim3(kWriteThreads), 0, stream, job);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ keep
// Rows of a request move towards its front, in place: row j comes from kept[j] >= j.  A round's rows are read and have arrived before any
// of them is written; what the writes cover are rows of the same round or before (a row that is still to be read, kept[i] for a later i,
// lies above kept[j] >= j), so that the next round's can be on their way by then.  A workgroup has CH 16-byte chunks of one head's rows,
// K's or V's, of a request in one cache: its rounds follow each other, but its chunks are its own.  Bound for accepted drafts by its chain
// of trips (lengths, list, table, rows: 16 requests in 32 layers 6.4 us), for long lists by the addresses of a workgroup's loads and
// stores, a lane's each for 16 bytes of a line: 4096 rows a round of 8 us (20001 of 32768 tokens of 8 heads of 64 in fp16 42 us, 1.9 TB/s; 51 with
// the next round's rows asked for after this one's are written).
struct PagedKeepJob {
    const int32_t *table, *q_start, *kv_lens, *kept, *n_kept;
    int64_t max_pages, max_kept;
    int row_bytes, shift;
    FastDiv by_h, by_splits;
    struct {
        char *K, *V;
        int64_t page_bytes;
        uint32_t n_pages;
    } cache[FEDRAG_KEEP_CACHES];
};

template <int THREADS, int CH>
FEDRAG_KERNEL __launch_bounds__(THREADS) void paged_keep_kernel(const PagedKeepJob j) {
    constexpr int kRows = THREADS / CH;  // rows that the workgroup's threads hold one chunk each of
    constexpr int kSteps = 4;
    const int b = (int)j.by_h.div(blockIdx.x), h = (int)(blockIdx.x - (uint32_t)b * j.by_h.d);
    const uint32_t layer = j.by_splits.div(blockIdx.y), split = blockIdx.y - layer * j.by_splits.d;
    const auto& cache = j.cache[layer];
    const int64_t page_bytes = cache.page_bytes;
    const uint32_t n_pages = cache.n_pages;
    const int row_bytes = j.row_bytes, shift = j.shift;
    char* const chunk = (blockIdx.z ? cache.V : cache.K) + ((int64_t)h << shift) * row_bytes + ((int)split * CH + threadIdx.x % CH) * 16;
    const int kv = j.kv_lens[b] < 0 ? 0 : j.kv_lens[b];
    const int64_t rows = (int64_t)j.q_start[b + 1] - j.q_start[b];
    const int n = rows < 0 ? 0 : rows < INT_MAX ? (int)rows : INT_MAX, base = kv - n;
    int64_t most = j.n_kept[b] < n ? j.n_kept[b] : n;
    most = most < j.max_kept ? most : j.max_kept;
    const uint32_t count = most > 0 ? (uint32_t)most : 0;
    const int32_t* const kept = j.kept + b * j.max_kept;
    const int32_t* const table = j.table + b * j.max_pages;
    const uint32_t end = j.max_pages << shift < kv ? (uint32_t)(j.max_pages << shift) : (uint32_t)kv;  // tokens that have a column
    auto page_of = [&](int token) { return (uint32_t)token < end ? table[(uint32_t)token >> shift] : -1; };
    auto place = [&](int page, int token) { return chunk + ((int64_t)page * page_bytes + (token & ((1 << shift) - 1)) * row_bytes); };
    // Four stages, each with the rows of a round in its arrays: the list, the table, the rows, and the writing.  Reading the rows of a round
    // before those of the round before are written is sound: they lie above all that these are written to.
    int k[kSteps], from_page[kSteps], to_page[kSteps], from[kSteps];
    char* to[kSteps];
    bool moves[kSteps];
    u32x4_t row[kSteps];
    const uint32_t step = threadIdx.x / CH;
    auto list = [&](uint32_t j0) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) k[u] = j0 + u * kRows + step < count ? kept[j0 + u * kRows + step] : -1;
    };
    auto pages_of = [&](uint32_t j0) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int i = (int)(j0 + u * kRows + step);
            const bool is = k[u] > i && k[u] < n;  // (a row that stays where it is has nothing to do)
            from[u] = base + k[u];
            from_page[u] = is ? page_of(base + k[u]) : -1;
            to_page[u] = is ? page_of(base + i) : -1;
        }
    };
    auto read = [&](uint32_t j0) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            moves[u] = (uint32_t)from_page[u] < n_pages && (uint32_t)to_page[u] < n_pages;
            to[u] = place(to_page[u], base + (int)(j0 + u * kRows + step));
            if (moves[u]) row[u] = *(const u32x4_t*)place(from_page[u], from[u]);
        }
    };
    constexpr uint32_t kRound = kSteps * kRows;
    list(0);
    pages_of(0);
    if (kRound < count) list(kRound);
    read(0);
    if (kRound < count) pages_of(kRound);
    for (uint32_t j0 = 0; j0 < count; j0 += kRound) {  // (count is at most INT_MAX)
        if (j0 + 2 * kRound < count) list(j0 + 2 * kRound);
        __builtin_amdgcn_s_waitcnt(0x0f70);  // this thread's chunks are here, and behind the barrier everybody's
        __syncthreads();
        char* old_to[kSteps];
        bool old_moves[kSteps];
        u32x4_t old[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            old_to[u] = to[u];
            old_moves[u] = moves[u];
            old[u] = row[u];
        }
        if (j0 + kRound < count) read(j0 + kRound);
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            if (old_moves[u]) *(u32x4_t*)old_to[u] = old[u];
        if (j0 + 2 * kRound < count) pages_of(j0 + 2 * kRound);
    }
}

hipError_t launch_paged_keep(const PagedKeep& k, hipStream_t stream) {
    PagedKeepJob j{};
    j.table = k.table;
    j.q_start = k.q_start;
    j.kv_lens = k.kv_lens;
    j.kept = k.kept;
    j.n_kept = k.n_kept;
    j.max_pages = k.max_pages;
    j.max_kept = k.max_kept;
    j.row_bytes = k.D * k.elem_bytes;
    j.shift = k.pages[0].shift;
    j.by_h = FastDiv(k.H);
    for (int i = 0; i < k.n_caches; ++i) {
        j.cache[i].K = (char*)k.pages[i].K;
        j.cache[i].V = (char*)k.pages[i].V;
        j.cache[i].page_bytes = k.pages[i].page_bytes;
        j.cache[i].n_pages = k.pages[i].n_pages;
    }
    // Accepted drafts: a wave for all chunks of a head's rows.  Long lists are a chain of steps, which workgroups of many threads and few
    // chunks make short: one to a workgroup (20001 of 32768 tokens, 8 heads of 64 in fp16, when one took 51 us: two chunks 59, all eight 255), or more while there
    // are two workgroups to a compute unit all the same.
    const int chunks = j.row_bytes / 16;
    const bool few = k.max_kept <= 64;
    int each = few ? chunks : 1;
    while (!few && each < chunks && (int64_t)k.B * k.H * 2 * k.n_caches * (chunks / each) > 2 * attn_target_wgs()) each *= 2;
    j.by_splits = FastDiv(chunks / each);
    const auto kernel = few ? (each == 8 ? paged_keep_kernel<64, 8> : each == 16 ? paged_keep_kernel<64, 16> : paged_keep_kernel<64, 32>)
                            : (each == 1 ? paged_keep_kernel<1024, 1> : each == 2 ? paged_keep_kernel<1024, 2> : each == 4 ? paged_keep_kernel<1024, 4> : each == 8 ? paged_keep_kernel<1024, 8>
                                         : each == 16 ? paged_keep_kernel<1024, 16> : paged_keep_kernel<1024, 32>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(k.B * k.H), (unsigned)(k.n_caches * (chunks / each)), 2), dim3(few ? 64 : 1024), 0, stream, j);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ trim
// The requests are taken 1024 at a time.  Their places on the stack are prefix sums of the pages that each gives back: entries of the table
// below 0 are none, so that the columns are looked at before any is written.  Up to 1024 columns are a thread's each, of the last
// workgroup; more are a wave's request by request, the columns of two requests in flight together: a workgroup counts what is before its
// share, and writes its share (the second time out of L2).  Nothing passes between workgroups, and the last one keeps the books.  64 requests
// of a page or none 4.6 us on the device, 3.9 in place; 256 that end at once, 63541 pages, 20.2, and in place, by one workgroup, 30.4: the last workgroup
// looks at the whole table by itself, 254 KB, and is bound by its trips, two requests' columns a wave at a time.
// (More columns in flight, or 16 bytes a lane: 33 to 42 us by one workgroup.)
constexpr int kTrimWaves = kMapThreads / kWave;
constexpr int kTrimMost = 16;  // workgroups
constexpr int kTrimAhead = 4;  // columns of a request that a lane has in flight

FEDRAG_KERNEL __launch_bounds__(kMapThreads) void paged_trim_kernel(PagedTrimJob j, int shift) {
    __shared__ MapPrefix waves[kTrimWaves];
    __shared__ uint32_t col_end[kMapThreads], found[kMapThreads];
    __shared__ int first_col[kMapThreads];
    __shared__ int range[kTrimWaves][2];
    __shared__ int flags;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const uint32_t wg = blockIdx.x, wgs = gridDim.x;
    const bool last = wg == wgs - 1;
    const int64_t max_pages = j.max_pages;
    const int count_in = *j.free_count;
    const uint32_t count = count_in < 0 ? 0 : (uint32_t)(count_in < j.n_free ? count_in : j.n_free);
    const uint32_t most = INT_MAX;
    uint32_t top = count;
    bool full = false;  // there is no room for all
    if (tid == 0) flags = (uint32_t)count_in == count ? 0 : FEDRAG_TRIM_BAD_LENGTH;
    auto below = [&](uint64_t lanes) { return (uint32_t)__builtin_popcountll(lanes & (((uint64_t)1 << lane) - 1)); };
    auto push = [&](uint32_t to, int id) {
        if (to < j.n_free) j.free_pages[to] = id;
    };
    for (int64_t b0 = 0; b0 < j.batch; b0 += kMapThreads) {
        __syncthreads();
        const int64_t b = b0 + tid;
        const int n_req = (int)(j.batch - b0 < kMapThreads ? j.batch - b0 : kMapThreads);
        uint32_t mine = 0;
        first_col[tid] = 0;
        found[tid] = 0;
        if (b < j.batch) {
            const int kv_in = j.kv_lens[b], kv = kv_in < 0 ? 0 : kv_in;
            int64_t len = j.n_kept[b];
            if (j.q_start) len += kv - ((int64_t)j.q_start[b + 1] - j.q_start[b]);
            const int64_t in = len;
            len = len < 0 ? 0 : (len < kv ? len : kv);
            if (in != len || kv_in < 0) atomicOr(&flags, FEDRAG_TRIM_BAD_LENGTH);
            const int64_t all = ((int64_t)kv + (1 << shift) - 1) >> shift, had = all < max_pages ? all : max_pages;
            const int64_t stay = (len + (1 << shift) - 1) >> shift;
            mine = had > stay ? (uint32_t)(had - stay) : 0;
            first_col[tid] = (int)stay;
            if (last) j.lens_out[b] = (int)len;
        }
        MapPrefix total;
        const MapPrefix p = map_scan(MapPrefix{mine, 0}, most, waves, &total);
        if (total.rows <= kMapThreads) {
            col_end[tid] = p.rows;
            __syncthreads();
            int id = -1;
            if ((uint32_t)tid < total.rows) {
                const int k = first_above(col_end, n_req, tid);
                id = j.block_table[(b0 + k) * max_pages + first_col[k] + (tid - (k == 0 ? 0 : col_end[k - 1]))];
            }
            const uint64_t pages = __builtin_amdgcn_ballot_w64(id >= 0);
            if (lane == 0) found[wave] = (uint32_t)__builtin_popcountll(pages);
            __syncthreads();
            uint32_t before = 0, sum = 0;
#pragma unroll
            for (int w = 0; w < kTrimWaves; ++w) {
                if (w == wave) before = sum;
                sum += found[w];
            }
            if (id >= 0 && last) push(top + before + below(pages), id);
            full = full || top + sum > (uint32_t)j.n_free;
            top = min(top + sum, (uint32_t)j.n_free);
            continue;
        }
        // This workgroup writes the pages of requests lo .. hi-1, an even share of the columns, and counts those before them, too (and those
        // behind them, if there are requests after these).
        auto up_to = [&](uint32_t w) {
            const uint32_t bound = (uint32_t)((uint64_t)total.rows * w / wgs);
            return __builtin_popcountll(__builtin_amdgcn_ballot_w64(b < j.batch && (w == wgs || p.rows - mine < bound)));
        };
        const int lo_here = up_to(wg), hi_here = up_to(wg + 1);
        if (lane == 0) {
            range[wave][0] = lo_here;
            range[wave][1] = hi_here;
        }
        col_end[tid] = mine;  // (how many, here)
        __syncthreads();
        int lo = 0, hi = 0;
#pragma unroll
        for (int w = 0; w < kTrimWaves; ++w) {
            lo += range[w][0];
            hi += range[w][1];
        }
        // f(request, a lane's entries of it from column c on, one every 64; -1: none)
        auto each = [&](int from, int end, auto f) {
            for (int k0 = from + wave; k0 < end; k0 += 2 * kTrimWaves) {
                const int k1 = k0 + kTrimWaves < end ? k0 + kTrimWaves : k0;
                const uint32_t n0 = col_end[k0], n1 = k1 != k0 ? col_end[k1] : 0;
                const int32_t* const row0 = j.block_table + (b0 + k0) * max_pages + first_col[k0];
                const int32_t* const row1 = j.block_table + (b0 + k1) * max_pages + first_col[k1];
                for (uint32_t c = 0; c < (n0 > n1 ? n0 : n1); c += kTrimAhead * kWave) {
                    int id[2][kTrimAhead];
#pragma unroll
                    for (int u = 0; u < kTrimAhead; ++u) {
                        const uint32_t at = c + u * kWave + lane;
                        id[0][u] = at < n0 ? row0[at] : -1;
                        id[1][u] = at < n1 ? row1[at] : -1;
                    }
                    f(k0, id[0]);
                    if (k1 != k0) f(k1, id[1]);
                }
            }
        };
        each(0, b0 + kMapThreads < j.batch ? n_req : hi, [&](int k, const int (&id)[kTrimAhead]) {
            uint32_t n = 0;
#pragma unroll
            for (int u = 0; u < kTrimAhead; ++u) n += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(id[u] >= 0));
            if (lane == 0) found[k] += n;
        });
        __syncthreads();
        MapPrefix all;
        const uint32_t here = found[tid];
        const MapPrefix q = map_scan(MapPrefix{here, 0}, most, waves, &all);
        found[tid] = top + (q.rows - here);  // where the request's next page goes
        __syncthreads();
        each(lo, hi, [&](int k, const int (&id)[kTrimAhead]) {
            uint32_t to = found[k];
            wave_lds_fence();  // (all lanes have it)
#pragma unroll
            for (int u = 0; u < kTrimAhead; ++u) {
                const uint64_t pages = __builtin_amdgcn_ballot_w64(id[u] >= 0);
                if (id[u] >= 0) push(to + below(pages), id[u]);
                to += (uint32_t)__builtin_popcountll(pages);
            }
            if (lane == 0) found[k] = to;
            wave_lds_fence();
        });
        full = full || top + all.rows > (uint32_t)j.n_free;
        top = min(top + all.rows, (uint32_t)j.n_free);
    }
    __syncthreads();
    if (tid == 0 && last) {
        *j.free_left = (int)top;
        *j.flags = flags | (full ? FEDRAG_TRIM_NO_ROOM : 0);
    }
}

hipError_t launch_paged_trim(const PagedTrimJob& job, hipStream_t stream) {
    // Lengths and a count that are written in place are one workgroup's work, as the others would still read them.  (256 requests of 300 to
    // 16000 tokens that end at once: 30.5 us by one, 22.8, 21.4, 20.6, 20.4 by 4, 8, 16, 32; of up to 900 17.5 and 12.0.)
    const bool in_place = job.lens_out == job.kv_lens || job.free_left == job.free_count;
    const int64_t shares = in_place ? 1 : (int64_t)job.batch * job.max_pages / kMapThreads;  // (of up to so many columns one reads each at once)
    const int wgs = shares < 1 ? 1 : shares < kTrimMost ? (int)shares : kTrimMost;
    hipLaunchKernelGGL(paged_trim_kernel, dim3((unsigned)wgs), dim3(kMapThreads), 0, stream, job, __builtin_ctz((unsigned)job.page_tokens));
    return hipGetLastError();
}

}  // namespace fedrag
