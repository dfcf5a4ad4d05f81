// Page tables of a batch of requests, kept on the device: a step's rows get pages, positions and slots from the requests' lengths,
// and pages behind the tokens that stay go back to the stack of free ones.
//
// Both kernels are sums over a flat list of page-table entries (request by request, ascending): the k-th missing entry takes
// free[count - 1 - k], the k-th entry that is given back goes to free[count + n - 1 - k].  One CTA walks the list, 1024 x 4 entries a
// trip; what bounds it is a trip's chain of dependent loads (entry, stack) and barriers, not bytes.  Rows are a second kernel over
// all SMs unless they are few.
#pragma once

#include "common.cuh"

namespace qift {

constexpr int kPtThreads = 1024, kPtWarps = kPtThreads / 32;
constexpr int kPtBatch = 2048;      // requests whose sums are held in shared memory at a time
constexpr int kPtPer = 4;           // entries of a thread in a trip
constexpr int kPtFewRows = 4096;    // rows that the one CTA fills in itself

struct PageTables {
    int32_t* table;                 // [R][max_pages]
    int32_t* free_pages;            // [num_pages] stack
    int32_t* free_count;            // [1]
    int R, max_pages, num_pages, page_tokens;
    __device__ __forceinline__ bool is_page(int v) const { return static_cast<unsigned>(v) < static_cast<unsigned>(num_pages); }
    __device__ __forceinline__ int free_now() const { return max(0, min(num_pages, *free_count)); }
};

struct PageBeginParams {
    PageTables t;
    const int32_t* rows;            // [R]
    const int32_t* first;           // [R]
    const int32_t* mask;            // [total][mask_words] or null
    int mask_words, total;
    int32_t* row_start;             // [R + 1]
    int32_t* position;              // [total]
    long long* slot;                // [total] or null
    int32_t* lost;                  // [1]
    int fill_rows;                  // the one CTA fills the rows in as well
};

struct PageEndParams {
    PageTables t;
    const int32_t* length;          // [R]
    const int32_t* shared;          // [R] or null
};

// Exclusive sum of v over the CTA's threads, and the total.  `tmp` holds kPtWarps values; two barriers.
template <typename T>
__device__ __forceinline__ T pt_scan(T v, T& total, T* tmp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T up = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += up;
    }
    __syncthreads();                // the last call's readers are done with tmp
    if (lane == 31) tmp[warp] = s;
    __syncthreads();
    T w = tmp[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T up = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += up;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const T before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return s - v + (warp ? before : T(0));
}

// The last i < n with start[i] <= x (ascending, start[0] <= x): of requests without entries, which start where the next one does,
// it finds the next one.
template <typename T>
__device__ __forceinline__ int pt_find(const T* start, int n, T x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int clamp_to_int(long long v) { return static_cast<int>(max(-1ll, min(v, 0x7fffffffll))); }

// Position and slot of a row of a call.
__device__ __forceinline__ void pt_row(const PageBeginParams& p, int row) {
    int position = -1;
    long long slot = -1;
    if (row < p.row_start[p.t.R]) {
        const int lo = pt_find(p.row_start, p.t.R, row);
        const int first = p.first[lo];
        const long long place = static_cast<long long>(first) + (row - p.row_start[lo]);
        const long long i = place / p.t.page_tokens;
        if (place >= 0 && i < p.t.max_pages) {
            const int page = p.t.table[static_cast<size_t>(lo) * p.t.max_pages + i];
            if (p.t.is_page(page)) slot = static_cast<long long>(page) * p.t.page_tokens + (place - i * p.t.page_tokens);
        }
        position = clamp_to_int(place);
        if (p.mask) {
            int seen = 0;
            const int32_t* m = p.mask + static_cast<size_t>(row) * p.mask_words;
            for (int w = 0; w < p.mask_words; ++w) seen += __popc(m[w]);
            position = clamp_to_int(static_cast<long long>(first) + max(seen - 1, 0));
        }
    }
    p.position[row] = position;
    if (p.slot) p.slot[row] = slot;
}

__global__ void __launch_bounds__(kPtThreads, 1)
pages_begin_kernel(const PageBeginParams p) {
    __shared__ int entry_start[kPtBatch];        // entries of the batch's requests before request i
    __shared__ int entry_lo[kPtBatch];           // the first entry of each that its rows fall into
    __shared__ long long tmp64[kPtWarps];
    __shared__ int tmp[kPtWarps];
    pdl_launch_dependents();
    pdl_wait();
    const PageTables& t = p.t;
    const int tid = threadIdx.x, P = t.page_tokens;
    const int have = t.free_now();
    const long long cap = static_cast<long long>(t.max_pages) * P;
    long long row_carry = 0, lost = 0;
    int taken = 0;                               // pages that entries have asked for so far
    for (int r0 = 0; r0 < t.R; r0 += kPtBatch) {
        const int nr = min(kPtBatch, t.R - r0);
        int entries = 0;                         // of the batch
        for (int b = 0; b < nr; b += kPtThreads) {
            const int r = r0 + b + tid;
            const bool on = b + tid < nr;
            const long long want = on ? max(0, p.rows[r]) : 0;
            long long sum;
            const long long start = row_carry + pt_scan(want, sum, tmp64);
            row_carry += sum;
            const long long begin = min(start, static_cast<long long>(p.total)), n = min(start + want, static_cast<long long>(p.total)) - begin;
            int lo = 0, e = 0;
            if (on) {
                p.row_start[r] = static_cast<int>(begin);
                const long long f = p.first[r];
                const long long a = max(f, 0ll), z = min(f + n, cap);
                if (z > a) lo = static_cast<int>(a / P), e = static_cast<int>((z + P - 1) / P) - lo;
                lost += want - max(0ll, z - a);
            }
            int esum;
            const int before = pt_scan(e, esum, tmp);
            if (on) entry_start[b + tid] = entries + before, entry_lo[b + tid] = lo;
            entries += esum;
        }
        __syncthreads();
        for (int k0 = 0; k0 < entries; k0 += kPtThreads * kPtPer) {
            size_t at[kPtPer];
            int owner[kPtPer], value[kPtPer], need = 0;
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                const int k = k0 + tid * kPtPer + j;
                value[j] = 0;
                if (k < entries) {
                    owner[j] = pt_find(entry_start, nr, k);
                    at[j] = static_cast<size_t>(r0 + owner[j]) * t.max_pages + entry_lo[owner[j]] + (k - entry_start[owner[j]]);
                    value[j] = t.table[at[j]];
                }
            }
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                const bool missing = k0 + tid * kPtPer + j < entries && !t.is_page(value[j]);
                value[j] = missing ? need : -1;
                need += missing;
            }
            int sum;
            const int before = taken + pt_scan(need, sum, tmp);
            taken += sum;
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                if (value[j] < 0) continue;
                const int k = before + value[j];
                int page = k < have ? t.free_pages[have - 1 - k] : -1;
                if (!t.is_page(page)) {
                    page = -1;
                    const int r = r0 + owner[j];
                    const long long f = p.first[r], n = min(static_cast<long long>(p.total) - p.row_start[r], static_cast<long long>(max(0, p.rows[r])));
                    const long long i = static_cast<long long>(at[j] - static_cast<size_t>(r) * t.max_pages);
                    lost += min(f + n, (i + 1) * P) - max(f, i * P);
                }
                t.table[at[j]] = page;
            }
        }
        __syncthreads();                         // entry_start is free again
    }
    long long all;
    pt_scan(lost, all, tmp64);
    if (tid == 0) {
        p.row_start[t.R] = static_cast<int>(min(row_carry, static_cast<long long>(p.total)));
        *t.free_count = have - min(taken, have);
        *p.lost = clamp_to_int(all);
    }
    if (p.fill_rows) {
        __syncthreads();                         // the table and row_start as this CTA has written them
        for (int row = tid; row < p.total; row += kPtThreads) pt_row(p, row);
    }
}

__global__ void __launch_bounds__(256)
pages_rows_kernel(const PageBeginParams p) {
    pdl_launch_dependents();
    pdl_wait();
    for (long long row = blockIdx.x * 256ll + threadIdx.x; row < p.total; row += gridDim.x * 256ll) pt_row(p, static_cast<int>(row));
}

__global__ void __launch_bounds__(kPtThreads, 1)
pages_end_kernel(const PageEndParams p) {
    __shared__ long long entry_start[kPtBatch];
    __shared__ int entry_lo[kPtBatch];
    __shared__ long long tmp64[kPtWarps];
    __shared__ int tmp[kPtWarps];
    pdl_launch_dependents();
    pdl_wait();
    const PageTables& t = p.t;
    const int tid = threadIdx.x, P = t.page_tokens;
    const int have = t.free_now();
    // the pages are counted first: the first of them is to end on top
    int back = 0;
    for (int pass = 0; pass < 2; ++pass) {
        int done = 0;
        for (int r0 = 0; r0 < t.R; r0 += kPtBatch) {
            const int nr = min(kPtBatch, t.R - r0);
            long long entries = 0;
            for (int b = 0; b < nr; b += kPtThreads) {
                const bool on = b + tid < nr;
                const int keep = on ? static_cast<int>(min((max(0, p.length[r0 + b + tid]) + static_cast<long long>(P) - 1) / P, static_cast<long long>(t.max_pages))) : 0;
                long long sum;
                const long long before = pt_scan(on ? static_cast<long long>(t.max_pages - keep) : 0ll, sum, tmp64);
                if (on) entry_start[b + tid] = entries + before, entry_lo[b + tid] = keep;
                entries += sum;
            }
            __syncthreads();
            for (long long k0 = 0; k0 < entries; k0 += kPtThreads * kPtPer) {
                int value[kPtPer], rank[kPtPer], found = 0;
#pragma unroll
                for (int j = 0; j < kPtPer; ++j) {
                    const long long k = k0 + tid * kPtPer + j;
                    value[j] = -1;
                    if (k < entries) {
                        const int o = pt_find(entry_start, nr, k);
                        const int i = entry_lo[o] + static_cast<int>(k - entry_start[o]);
                        int32_t* at = t.table + static_cast<size_t>(r0 + o) * t.max_pages + i;
                        value[j] = *at;
                        if (pass == 1) *at = -1;
                        if (p.shared && i < p.shared[r0 + o]) value[j] = -1;
                    }
                    rank[j] = found;
                    if (t.is_page(value[j])) ++found;
                }
                int sum;
                const int before = done + pt_scan(found, sum, tmp);
                done += sum;
                if (pass == 1) {
#pragma unroll
                    for (int j = 0; j < kPtPer; ++j)
                        if (t.is_page(value[j])) {
                            const long long to = static_cast<long long>(have) + back - 1 - (before + rank[j]);
                            if (to < t.num_pages) t.free_pages[to] = value[j];
                        }
                }
            }
            __syncthreads();
        }
        back = done;
    }
    if (tid == 0) *t.free_count = static_cast<int>(min(static_cast<long long>(have) + back, static_cast<long long>(t.num_pages)));
}

}  // namespace qift
