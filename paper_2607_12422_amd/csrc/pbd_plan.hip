// Page tables and slot maps of packed rows, built from the requests' lengths on the
// device, and pages given back.
//
// The free pages are a stack.  Who gets which is a prefix sum: sequence b needs
// need_b = ceil((len_b + n_b) / P) - pages_b pages, and its i-th is the one that many
// (need_0 + .. + need_{b-1} + i) below the top, if the sum up to its own is there.  One
// work-group takes the sums, 1024 sequences at a time, and writes the tables; the rows
// follow, in the same launch where there are few.  Nothing here but waits (lengths, sums,
// page ids, table, rows: each for the one before): a plan of 17 rows takes 6.7 us, of 200
// sequences and 40100 rows 10.2 and 3.9 for the rows, their releases 5.7 and 9.6.
#include "pbd_launch.h"
#include "pbd_rows.h"

#include <algorithm>

namespace pbd {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;

__device__ __forceinline__ void raise(int* status, int bit) {
    if (status) atomicOr(status, bit);
}

// Inclusive sums over the work-group, and their total; ends with the shared words free again.
__device__ __forceinline__ long long group_scan(long long x, long long* s_wave, long long& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const long long y = __shfl_up(x, d, 64);
        if (lane >= d) x += y;
    }
    if (lane == 63) s_wave[wave] = x;
    __syncthreads();
    long long before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += s_wave[w];
        total += s_wave[w];
    }
    __syncthreads();
    return x + before;
}

// The first of n ascending sums that exceeds i (one does).
__device__ __forceinline__ int first_above(const int* sums, int n, int i) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] > i) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__device__ __forceinline__ int clamp31(long long x) { return (int)min(x, 0x7fffffffll); }

// One packed row: its sequence, position and slot.
__device__ __forceinline__ void put_row(const PagePlanArgs& a, int r, int b) {
    int slot = -1, at = 0;
    if (b >= 0) {
        const int i = r - a.row_start[b], len = a.lens[b];
        if (a.row_pos) at = a.pos[b] + i;
        if (a.new_lens[b] != len) {                  // (it has rows: equal only where it was skipped)
            const int s = len + i;
            const int id = a.table[(size_t)b * a.table_width + (s >> a.page_bits)];
            // (a page that the sequence had: shifted, an id past the pool may be another page's slot)
            if (id >= 0 && id < a.n_pages) slot = id << a.page_bits | (s & ((1 << a.page_bits) - 1));
            else raise(a.status, PBD_STATUS_PAGE);
        }
    }
    a.slot_map[r] = slot;
    if (a.row_seq) a.row_seq[r] = b;
    if (a.row_pos) a.row_pos[r] = at;
}

// The last of the sequences lo .. hi whose rows begin at or before row r.
__device__ __forceinline__ int owner(const int* row_start, int lo, int hi, int r) {
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (row_start[mid] <= r) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__global__ __launch_bounds__(THREADS) void k_page_plan(PagePlanArgs a) {
    __shared__ long long s_wave[WAVES];
    __shared__ int s_sum[THREADS], s_have[THREADS], s_taken;
    const int P = 1 << a.page_bits, tid = threadIdx.x;
    const int tiles = (a.batch + THREADS - 1) / THREADS;
    int f = *a.n_free;
    if (f < 0 || f > a.n_pages) {
        if (tid == 0) raise(a.status, PBD_STATUS_CAPACITY);
        f = 0;
    }
    if (tid == 0) s_taken = 0;
    int len = 0, n = 0, have = 0;
    long long need = 0, rows_to = 0, need_to = 0, all_rows = 0, all_need = 0;    // sums with the thread's own, and of the tile
    bool valid = false, served = false;
    long long rows_before = 0, need_before = 0;
    auto sums = [&](int tile) {
        const int b = tile * THREADS + tid;
        len = n = have = 0;
        valid = false;
        if (b < a.batch) {
            len = a.lens[b];
            n = a.n_new[b];
            have = a.seq_pages[b];
            valid = len >= 0 && n >= 0 && have >= 0 && have <= a.table_width && len <= (long long)have * P &&
                    (long long)len + n <= (long long)a.table_width * P;
        }
        rows_to = rows_before + group_scan(max(n, 0), s_wave, all_rows);
        valid = valid && rows_to <= a.max_rows;
        need = valid ? max(0ll, ((long long)len + n + P - 1) / P - have) : 0;
        need_to = need_before + group_scan(need, s_wave, all_need);
        served = valid && (need == 0 || need_to <= f);
    };
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        sums(t);
        if (served && need > 0) atomicMax(&s_taken, (int)need_to);
        if (tiles > 1) {
            rows_before += all_rows;
            need_before += all_need;
        }
    }
    __syncthreads();
    int taken = s_taken;
    bool bad = false;
    for (int i = tid; i < taken; i += THREADS) {
        const int id = a.free_pages[f - 1 - i];
        bad |= id < 0 || id >= a.n_pages;
    }
    if (__syncthreads_or(bad)) {
        // a stack that holds no pages serves nobody
        if (tid == 0) raise(a.status, PBD_STATUS_PAGE);
        f = taken = 0;
        served = valid && need == 0;
    }
    rows_before = need_before = 0;
    for (int t = 0; t < tiles; ++t) {
        if (tiles > 1) sums(t);
        const int b = t * THREADS + tid;
        const int in_tile = clamp31(need_to - need_before);
        s_sum[tid] = in_tile;
        s_have[tid] = have;
        if (b < a.batch) {
            const long long first = rows_to - max(n, 0);
            a.row_start[b] = (int)min(first, (long long)a.max_rows);
            if (b == a.batch - 1) a.row_start[a.batch] = (int)min(rows_to, (long long)a.max_rows);
            a.new_lens[b] = served ? len + n : len;
            if (served && need > 0) a.seq_pages[b] = have + (int)need;
            if (!served) raise(a.status, PBD_STATUS_CAPACITY);
        }
        __syncthreads();
        // the tile's new pages, one to a thread
        const int pages = (int)max(0ll, min((long long)taken - need_before, all_need));
        for (int i = tid; i < pages; i += THREADS) {
            const int q = first_above(s_sum, THREADS, i), p = s_have[q] + i - (q > 0 ? s_sum[q - 1] : 0);
            a.table[(size_t)(t * THREADS + q) * a.table_width + p] = a.free_pages[f - 1 - (need_before + i)];
        }
        __syncthreads();
        rows_before += all_rows;
        need_before += all_need;
    }
    if (tid == 0 && taken > 0) *a.n_free = f - taken;
    if (!a.rows_here) return;
    const int total = (int)min(rows_before, (long long)a.max_rows);
    for (int r = tid; r < a.max_rows; r += THREADS) put_row(a, r, r < total ? owner(a.row_start, 0, a.batch - 1, r) : -1);
}

// The rows of larger plans: a work-group finds the sequences of its first and its last
// row, 64 candidates at a time, and a row looks between them.
__global__ __launch_bounds__(256) void k_page_rows(PagePlanArgs a) {
    const int lane = threadIdx.x & 63, r = blockIdx.x * 256 + threadIdx.x;
    const int total = a.row_start[a.batch], first = blockIdx.x * 256, last = min(first + 255, total - 1);
    int b = -1;
    if (first < total) {
        int ends[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int want = e ? last : first;
            int lo = 0, hi = a.batch;
            while (hi - lo > 1) {
                const int step = (hi - lo + 63) / 64;
                const long long at = (long long)lo + (long long)lane * step;
                const bool below = at < hi && (lane == 0 || a.row_start[min(at, (long long)a.batch)] <= want);
                const int cnt = __popcll(__ballot(below));
                lo += (cnt - 1) * step;
                hi = min(hi, lo + step);
            }
            ends[e] = lo;
        }
        if (r < total) b = owner(a.row_start, ends[0], ends[1], r);
    }
    if (r < a.max_rows) put_row(a, r, b);
}

__global__ __launch_bounds__(THREADS) void k_page_release(PageReleaseArgs a) {
    __shared__ long long s_wave[WAVES];
    __shared__ int s_sum[THREADS], s_have[THREADS], s_bad[THREADS];
    const int P = 1 << a.page_bits, tid = threadIdx.x;
    const int tiles = (a.batch + THREADS - 1) / THREADS;
    const int f = *a.n_free;
    int have = 0, stay = 0;
    long long gone = 0, gone_to = 0, all = 0, before = 0;
    auto sums = [&](int tile, bool report) {
        const int b = tile * THREADS + tid;
        have = stay = 0;
        gone = 0;
        bool bad = false;
        if (b < a.batch) {
            have = a.seq_pages[b];
            const int keep = a.keep[b];
            bad = have < 0 || have > a.table_width || keep < 0;
            if (!bad) {
                stay = (int)min((long long)have, ((long long)keep + P - 1) / P);
                gone = have - stay;
            }
            if (bad && report) raise(a.status, PBD_STATUS_CAPACITY);
        }
        // no page of a sequence goes unless all that would are pages
        s_sum[tid] = clamp31(group_scan(gone, s_wave, all));
        s_have[tid] = stay;
        s_bad[tid] = 0;
        __syncthreads();
        for (int i = tid; i < clamp31(all); i += THREADS) {
            const int q = first_above(s_sum, THREADS, i), p = s_have[q] + i - (q > 0 ? s_sum[q - 1] : 0);
            const int id = a.table[(size_t)(tile * THREADS + q) * a.table_width + p];
            if (id < 0 || id >= a.n_pages) s_bad[q] = 1;
        }
        __syncthreads();
        if (s_bad[tid]) {
            gone = 0;
            if (report) raise(a.status, PBD_STATUS_PAGE);
        }
        gone_to = before + group_scan(gone, s_wave, all);
        s_sum[tid] = clamp31(gone_to - before);
        __syncthreads();
    };
    for (int t = 0; t < tiles; ++t) {
        sums(t, true);
        before += all;
    }
    const long long total = before;
    if (f < 0 || f + total > a.n_pages) {
        if (tid == 0) raise(a.status, PBD_STATUS_CAPACITY);      // (pages given back twice)
        return;
    }
    if (total == 0) return;
    before = 0;
    for (int t = 0; t < tiles; ++t) {
        if (tiles > 1) sums(t, false);
        // the last page of the last sequence first, so that a plan's pages return to where it took them from
        for (int i = tid; i < (int)all; i += THREADS) {
            const int q = first_above(s_sum, THREADS, i), j = i - (q > 0 ? s_sum[q - 1] : 0), cnt = s_sum[q] - (q > 0 ? s_sum[q - 1] : 0);
            int* e = a.table + (size_t)(t * THREADS + q) * a.table_width + s_have[q] + j;
            a.free_pages[f + (total - before - s_sum[q]) + (cnt - 1 - j)] = *e;
            *e = -1;
        }
        if (gone > 0) a.seq_pages[t * THREADS + tid] = stay;
        __syncthreads();
        before += all;
    }
    if (tid == 0) *a.n_free = (int)(f + total);
}

}  // namespace

// Rows that the scan's work-group does itself: a launch less, for a pass over its rows
// that one CU makes 1024 at a time (plan and release, us, in one launch and in two: 17
// rows 14.0 and 17.4, 1024 15.7 and 18.7, 4096 19.5 and 19.0, 16384 37 and 19).
constexpr int ROWS_HERE = 3584;

hipError_t launch_page_plan(const PagePlanArgs& args, hipStream_t st) {
    PagePlanArgs a = args;
    a.rows_here = a.max_rows <= ROWS_HERE;
    PBD_LAUNCH(k_page_plan, dim3(1), dim3(THREADS), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.rows_here) return e;
    PBD_LAUNCH(k_page_rows, dim3((a.max_rows + 255) / 256), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_page_release(const PageReleaseArgs& a, hipStream_t st) {
    PBD_LAUNCH(k_page_release, dim3(1), dim3(THREADS), 0, st, a);
    return hipGetLastError();
}

}  // namespace pbd
