// Page tables of a batch of requests, kept on the device: a step's rows get pages, positions and slots from the requests' lengths,
// and pages behind the tokens that stay go back to the stack of free ones.
//
// Both are sums over a flat list of page-table entries (request by request, ascending): the k-th missing entry takes
// free[count - 1 - k]; a page that is given back goes behind the stack's top and all pages given back after it, so that list is walked from its
// end and needs no second pass.  What bounds them is a chain of dependent loads and barriers (rows, sums over requests, entries, sums over
// entries, the stack), not bytes: one CTA of 256 threads where that covers the list, clusters of eight CTAs of 1024 that exchange
// their sums through distributed shared memory otherwise, 4 entries a thread and trip.  Many rows are a second kernel over all SMs.
// Begin and end together: 64 single tokens behind up to 8000 10.7 us (15.4 in the first form), 192 trees of up to 64 behind
// 2000 18.5, 256 prompts, 580 000 rows, 23.2 (60).  Cold, under the profiler, the last took 12.1 (begin), 9.5 (rows) and 10.5
// us (end); what the first and the last of them wait for most is one another's warps, at barriers.
#pragma once

#include "common.cuh"

namespace qift {

constexpr int kPtPer = 4;           // entries of a thread in a trip
constexpr int kPtBatch = 2048;      // requests whose sums are held in shared memory at a time
constexpr int kPtCluster = 8;
constexpr int kPtFewThreads = 256, kPtManyThreads = 1024;
constexpr int kPtMaxRequests = 1 << 30;   // sums of two of their numbers stay within 32 bits
constexpr int kPtFewRows = 1024;    // rows that the first kernel fills in itself

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
    int fill_rows;                  // the first kernel fills the rows in as well (one CTA)
};

struct PageEndParams {
    PageTables t;
    const int32_t* length;          // [R]
    const int32_t* shared;          // [R] or null
};

// Exclusive sum of v over the CTA's threads, and the total.  `tmp` holds a value per warp; two barriers.
template <typename T>
__device__ __forceinline__ T pt_scan(T v, T& total, T* tmp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    T s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T up = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += up;
    }
    __syncthreads();                // the last call's readers are done with tmp
    if (lane == 31) tmp[warp] = s;
    __syncthreads();
    T w = lane < warps ? tmp[lane] : T(0);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T up = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += up;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const T before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return s - v + (warp ? before : T(0));
}

// Exclusive sum over the cluster: of the CTAs before this one (after it, if `behind`), and of all.  Trips alternate between two buffers, so one
// cluster barrier a trip is enough: a CTA that writes a buffer again has met everybody in between.
template <int CL>
__device__ __forceinline__ int pt_cluster(int mine, int& total, int (*counts)[kPtCluster], int parity, bool behind) {
    if constexpr (CL == 1) {
        total = mine;
        return 0;
    } else {
        const uint32_t rank = cluster_ctarank();
        if (threadIdx.x < CL) {
            uint32_t at;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&counts[parity][rank])), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(at), "r"(mine) : "memory");
        }
        cluster_sync_all();
        int before = 0;
        total = 0;
#pragma unroll
        for (int i = 0; i < CL; ++i) {
            const int c = counts[parity][i];
            total += c;
            if (behind ? i > static_cast<int>(rank) : i < static_cast<int>(rank)) before += c;
        }
        return before;
    }
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

// Position and slot of a row of request r, or of nobody's (r < 0).
__device__ __forceinline__ void pt_row(const PageBeginParams& p, int row, int r) {
    int position = -1;
    long long slot = -1;
    if (r >= 0) {
        const int first = p.first[r];
        const long long place = static_cast<long long>(first) + (row - p.row_start[r]);
        if (place >= 0 && place < static_cast<long long>(p.t.max_pages) * p.t.page_tokens) {
            const unsigned i = place <= 0x7fffffffll ? static_cast<unsigned>(place) / p.t.page_tokens : static_cast<unsigned>(place / p.t.page_tokens);
            const int page = p.t.table[static_cast<size_t>(r) * p.t.max_pages + i];
            if (p.t.is_page(page)) slot = static_cast<long long>(page) * p.t.page_tokens + (place - static_cast<long long>(i) * p.t.page_tokens);
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

template <int CL>
__global__ void __launch_bounds__(kPtManyThreads, 1)
pages_begin_kernel(const PageBeginParams p) {
    __shared__ int entry_start[kPtBatch];        // entries of the batch's requests before request i
    __shared__ int entry_lo[kPtBatch];           // the first entry of each that its rows fall into
    __shared__ int kept[kPtBatch];               // its rows that the call has room for
    __shared__ long long tmp64[32];
    __shared__ int tmp[32];
    __shared__ int counts[2][kPtCluster];
    pdl_launch_dependents();
    if constexpr (CL > 1) cluster_sync_all();    // every CTA of the cluster runs before anything is written to its shared memory
    pdl_wait();
    const PageTables& t = p.t;
    const int tid = threadIdx.x, threads = blockDim.x, P = t.page_tokens;
    const int rank = CL > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int have = t.free_now();
    const long long cap = static_cast<long long>(t.max_pages) * P;
    long long row_carry = 0, lost = 0;
    int taken = 0, trip = 0;                     // pages that entries have asked for so far
    for (int r0 = 0; r0 < t.R; r0 += kPtBatch) {
        const int nr = min(kPtBatch, t.R - r0);
        int entries = 0;                         // of the batch; every CTA works the sums over the requests out for itself
        for (int b = 0; b < nr; b += threads) {
            const int r = r0 + b + tid;
            const bool on = b + tid < nr;
            const long long want = on ? max(0, p.rows[r]) : 0, f = on ? p.first[r] : 0;
            auto span = [&](long long n, int& lo) {     // entries that n rows from f on fall into
                const long long a = max(f, 0ll), z = min(f + n, cap);
                lo = z > a ? static_cast<int>(a / P) : 0;
                return z > a ? static_cast<int>((z + P - 1) / P) - lo : 0;
            };
            long long sum;
            const long long start = row_carry + pt_scan(want, sum, tmp64);
            const long long begin = min(start, static_cast<long long>(p.total)), n = min(start + want, static_cast<long long>(p.total)) - begin;
            int lo;
            const int e = span(n, lo);
            row_carry += sum;
            int esum;
            const int ebefore = pt_scan(e, esum, tmp);
            if (on) {
                if (rank == 0) {
                    p.row_start[r] = static_cast<int>(begin);
                    lost += want - max(0ll, min(f + n, cap) - max(f, 0ll));
                }
                entry_start[b + tid] = entries + ebefore, entry_lo[b + tid] = lo, kept[b + tid] = static_cast<int>(n);
            }
            entries += esum;
        }
        __syncthreads();
        for (int k0 = 0; k0 < entries; k0 += CL * threads * kPtPer, ++trip) {
            size_t at[kPtPer];
            int owner[kPtPer], value[kPtPer], need = 0;
            const int mine = k0 + (rank * threads + tid) * kPtPer;
            int o = mine < entries ? pt_find(entry_start, nr, mine) : 0;
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                const int k = mine + j;
                value[j] = 0;
                if (k < entries) {
                    while (o + 1 < nr && entry_start[o + 1] <= k) ++o;
                    owner[j] = o;
                    at[j] = static_cast<size_t>(r0 + o) * t.max_pages + entry_lo[o] + (k - entry_start[o]);
                    value[j] = t.table[at[j]];
                }
            }
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                const bool missing = mine + j < entries && !t.is_page(value[j]);
                value[j] = missing ? need : -1;
                need += missing;
            }
            int sum, all;
            const int in_cta = pt_scan(need, sum, tmp);
            const int before = taken + pt_cluster<CL>(sum, all, counts, trip & 1, false) + in_cta;
            taken += all;
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                if (value[j] < 0) continue;
                const int k = before + value[j];
                int page = k < have ? t.free_pages[have - 1 - k] : -1;
                if (!t.is_page(page)) {
                    page = -1;
                    const int r = r0 + owner[j];
                    const long long f = p.first[r], n = kept[owner[j]], i = static_cast<long long>(at[j] - static_cast<size_t>(r) * t.max_pages);
                    lost += min(f + n, (i + 1) * P) - max(f, i * P);
                }
                t.table[at[j]] = page;
            }
        }
        __syncthreads();                         // entry_start is free again
    }
    long long all;
    pt_scan(lost, all, tmp64);
    if constexpr (CL > 1) {
        // the first CTA adds the others' up
        __shared__ long long sums[kPtCluster];
        if (tid == 0) {
            uint32_t to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(&sums[rank])), "r"(0));
            asm volatile("st.shared::cluster.s64 [%0], %1;" ::"r"(to), "l"(all) : "memory");
        }
        cluster_sync_all();                      // (and nobody leaves before the last write to another's shared memory)
        all = 0;
        if (rank == 0 && tid == 0)
            for (int i = 0; i < CL; ++i) all += sums[i];
    }
    if (rank == 0 && tid == 0) {
        p.row_start[t.R] = static_cast<int>(min(row_carry, static_cast<long long>(p.total)));
        *t.free_count = have - min(taken, have);
        *p.lost = clamp_to_int(all);
    }
    if (CL == 1 && p.fill_rows) {
        __syncthreads();                         // the table and row_start as this CTA has written them
        const int end = p.row_start[t.R];
        for (int row = tid; row < p.total; row += threads) pt_row(p, row, row < end ? pt_find(p.row_start, t.R, row) : -1);
    }
}

// A warp takes 128 rows at a time: requests are looked for once where all of them belong to one.
__global__ void __launch_bounds__(256)
pages_rows_kernel(const PageBeginParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, end = p.row_start[p.t.R];
    const long long step = static_cast<long long>(gridDim.x) * 8 * 128;
    for (long long row0 = (static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5)) * 128; row0 < p.total; row0 += step) {
        const int last = static_cast<int>(min(row0 + 127, static_cast<long long>(end) - 1));
        const int lo = row0 < end ? pt_find(p.row_start, p.t.R, static_cast<int>(row0)) : -1;
        const bool one = lo >= 0 && p.row_start[lo + 1] > last;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long row = row0 + j * 32 + lane;
            if (row >= p.total) break;
            int r = -1;
            if (row < end) r = one ? lo : lo + pt_find(p.row_start + lo, p.t.R - lo, static_cast<int>(row));
            pt_row(p, static_cast<int>(row), r);
        }
    }
}

template <int CL>
__global__ void __launch_bounds__(kPtManyThreads, 1)
pages_end_kernel(const PageEndParams p) {
    __shared__ int entry_start[kPtBatch];
    __shared__ int entry_lo[kPtBatch];
    __shared__ int tmp[32];
    __shared__ int counts[2][kPtCluster];
    pdl_launch_dependents();
    if constexpr (CL > 1) cluster_sync_all();
    pdl_wait();
    const PageTables& t = p.t;
    const int tid = threadIdx.x, threads = blockDim.x, P = t.page_tokens;
    const int rank = CL > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int have = t.free_now();
    long long back = 0;                          // pages given back so far: those behind, since the list is walked from its end
    int trip = 0;
    const int batches = (t.R + kPtBatch - 1) / kPtBatch;
    for (int batch = batches - 1; batch >= 0; --batch) {
        const int r0 = batch * kPtBatch, nr = min(kPtBatch, t.R - r0);
        int entries = 0;                         // (R * max_pages < 2^31)
        for (int b = 0; b < nr; b += threads) {
            const bool on = b + tid < nr;
            const int keep = on ? static_cast<int>(min((max(0, p.length[r0 + b + tid]) + static_cast<long long>(P) - 1) / P, static_cast<long long>(t.max_pages))) : 0;
            int sum;
            const int before = pt_scan(on ? t.max_pages - keep : 0, sum, tmp);
            if (on) entry_start[b + tid] = entries + before, entry_lo[b + tid] = keep;
            entries += sum;
        }
        __syncthreads();
        const int span = CL * threads * kPtPer;
        for (long long k0 = (static_cast<long long>(entries) - 1) / span * span; entries > 0 && k0 >= 0; k0 -= span, ++trip) {
            int value[kPtPer], found = 0;
            const long long mine = k0 + (rank * threads + tid) * kPtPer;
            int o = mine < entries ? pt_find(entry_start, nr, static_cast<int>(mine)) : 0;
            int32_t* at[kPtPer];
            bool give[kPtPer];
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                const long long k = mine + j;
                value[j] = -1, at[j] = nullptr, give[j] = true;
                if (k < entries) {
                    while (o + 1 < nr && entry_start[o + 1] <= k) ++o;
                    const int i = entry_lo[o] + static_cast<int>(k - entry_start[o]);
                    at[j] = t.table + static_cast<size_t>(r0 + o) * t.max_pages + i;
                    value[j] = *at[j];
                    give[j] = !p.shared || i >= p.shared[r0 + o];
                }
            }
#pragma unroll
            for (int j = 0; j < kPtPer; ++j) {
                if (at[j] && value[j] != -1) *at[j] = -1;
                if (!give[j]) value[j] = -1;
                found += t.is_page(value[j]);
            }
            int sum, all;
            const int in_cta = pt_scan(found, sum, tmp);
            long long behind = back + pt_cluster<CL>(sum, all, counts, trip & 1, true) + (sum - in_cta);   // this thread's own and all after them
            back += all;
#pragma unroll
            for (int j = 0; j < kPtPer; ++j)
                if (t.is_page(value[j])) {
                    const long long to = have + --behind;
                    if (to < t.num_pages) t.free_pages[to] = value[j];
                }
        }
        __syncthreads();
    }
    if constexpr (CL > 1) cluster_sync_all();    // nobody leaves before the last write to another's shared memory, and all have read the count
    if (rank == 0 && tid == 0) *t.free_count = static_cast<int>(min(have + back, static_cast<long long>(t.num_pages)));
}

}  // namespace qift
