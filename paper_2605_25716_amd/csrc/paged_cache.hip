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

}  // namespace fedrag
