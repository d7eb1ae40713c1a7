// Pages of the paged cache that requests share: page tables forked and released, pages reserved for new tokens (a shared page is copied before it is written) and live pages
// moved together.  refs[page] counts the entries of the caller's page tables that hold a page, 0: free.
//
// Everything is decided on the device from refs, tables and lengths, so a captured step follows them.  Who gets which page does not depend on the order in which threads
// come: needs are numbered in the order of sequences and columns, free pages in their own, and need j gets free page j.
//
// Bound: latencies.  The decisions are one CTA's (a scan over refs and a scan over the columns that new tokens touch; what they read is a few hundred kilobytes), the
// copying of bytes, bound by HBM, is a second launch's over all SMs (us: 4.5 to decide what moves of 4000 pages, 6 what 256 sequences get of 3300, 2 the launch behind it).
#pragma once
#include <cuda_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "paged.cuh"

namespace ql {

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;

__device__ __forceinline__ bool in_pool(int page, int n_pages) { return page >= 0 && page < n_pages; }
// Pages that hold n tokens of a table of `width` columns.
__device__ __forceinline__ int pages_of(int n, int log2_page, int width) { return n <= 0 ? 0 : min(((n - 1) >> log2_page) + 1, width); }

struct PagedForkParams {
    const int32_t* table;
    const int32_t* parents;
    const int32_t* lengths;
    int32_t* children;
    int32_t* refs;
    int64_t table_ld, children_ld;
    int32_t B, width, n_pages, log2_page;
};

// Row y of the children: the pages of the first lengths[y] tokens of its parent's row; each has one holder more.
__global__ void __launch_bounds__(256) paged_fork_kernel(const PagedForkParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int j = blockIdx.x * 256 + threadIdx.x, i = blockIdx.y;
    if (j >= p.width) return;
    const int parent = p.parents[i], n = pages_of(p.lengths[i], p.log2_page, p.width);
    int page = parent >= 0 && parent < p.B && j < n ? p.table[parent * p.table_ld + j] : -1;
    if (!in_pool(page, p.n_pages)) page = -1;
    p.children[i * p.children_ld + j] = page;
    if (page >= 0) atomicAdd(p.refs + page, 1);
}

struct PagedReleaseParams {
    int32_t* table;
    const int32_t* rows;
    const int32_t* keep;         // may be null: nothing is kept
    int32_t* refs;
    int64_t table_ld;
    int32_t B, width, n_pages, log2_page;
};

// Row rows[y] gives back its pages behind its first keep[y] tokens.  An entry is taken once, whichever thread comes to it first: a row may be named twice.
__global__ void __launch_bounds__(256) paged_release_kernel(const PagedReleaseParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int j = blockIdx.x * 256 + threadIdx.x, row = p.rows[blockIdx.y];
    if (j >= p.width || row < 0 || row >= p.B || (p.keep && j < pages_of(p.keep[blockIdx.y], p.log2_page, p.width))) return;
    const int page = atomicExch(p.table + row * p.table_ld + j, -1);
    if (in_pool(page, p.n_pages)) atomicSub(p.refs + page, 1);
}

// Exclusive sum over the CTA's threads and, in *total, the whole sum (64 bits where q_start may name rows more than once, against the rules).  Every thread takes part; `sums` may be used again by the next call.
template <typename T>
__device__ __forceinline__ T plan_scan(T v, T* total, T* sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T run = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T u = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += u;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = run;
    __syncthreads();
    T before = lane < kPlanWarps ? sums[lane] : 0;
    T all = before;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T u = __shfl_up_sync(0xffffffffu, all, o);
        if (lane >= o) all += u;
    }
    *total = __shfl_sync(0xffffffffu, all, 31);
    before = __shfl_sync(0xffffffffu, all - before, warp);
    return run - v + before;
}

// The pages of a warp: [lo, hi), whole groups of 128.
__device__ __forceinline__ void plan_share(int n_pages, int* lo, int* hi)
{
    const int warp = threadIdx.x >> 5, per = (((n_pages + 127) >> 7) + kPlanWarps - 1) / kPlanWarps;
    *lo = (int)min((int64_t)warp * per << 7, (int64_t)n_pages);
    *hi = (int)min((int64_t)*lo + ((int64_t)per << 7), (int64_t)n_pages);
}
// For the pages base + lane, base + 32 + lane, ... + 96 + lane of a warp's share: bit k of the result is set if refs of the k-th is above zero; bits 8 + k: the page lies in the share.
__device__ __forceinline__ uint32_t plan_live(const int32_t* refs, int base, int hi)
{
    uint32_t r = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int page = base + 32 * k + (threadIdx.x & 31);
        if (page < hi) r |= (refs[page] > 0 ? 1u : 0u) << k | 256u << k;
    }
    return r;
}

// need, free_list, copies: the workspace, n_pages entries each.
struct PagedReserveParams {
    PagedBatch batch;
    int32_t* table;
    int32_t* refs;
    int32_t* missing;            // pages that the pool is short of
    int4* need;                  // sequence, column, the page that is replaced (-1: none), blocks of it that hold older tokens
    int32_t* free_list;
    int4* copies;                // from, to, blocks of each head
    int32_t* n_copies;
};

__global__ void __launch_bounds__(kPlanThreads) paged_reserve_kernel(const PagedReserveParams p)
{
    extern __shared__ int pre[];                                         // [B + 1] columns before sequence b, [B] the first column of it
    __shared__ int sums[kPlanWarps], copied;
    __shared__ long long wide_sums[kPlanWarps];
    const PagedBatch& bt = p.batch;
    const int tid = threadIdx.x, lane = tid & 31, B = bt.B, log2_page = bt.log2_blocks + 4, n_pages = bt.n_pages;
    int* first = pre + B + 1;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) { copied = 0; pre[0] = 0; }
    // ---- the columns that new tokens come to
    long long columns = 0;
    for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        int n = 0, t0;
        long long all;
        if (b < B) {
            const int rows = paged_rows(bt, b, &t0), len = bt.kv_len[b];
            if (rows > 0 && len > 0) {
                const int c0 = max((int64_t)len - rows, (int64_t)0) >> log2_page;
                first[b] = c0;
                n = max(pages_of(len, log2_page, bt.table_width) - c0, 0);
            }
        }
        const long long before = plan_scan((long long)n, &all, wide_sums);
        if (b < B) pre[b + 1] = (int)(columns + before + n);
        columns += all;
    }
    if (columns > INT_MAX) {                                             // (rows named more than once: they lie in T / page_size + 2 B columns at most)
        if (tid == 0) { *p.missing = INT_MAX; *p.n_copies = 0; }
        return;
    }
    __syncthreads();
    // ---- those without a page of their own, in order
    int needs = 0;
    for (int64_t k0 = 0; k0 < columns; k0 += kPlanThreads) {
        const int k = (int)min(k0 + tid, (int64_t)INT_MAX);
        int b = 0, c = 0, page = -1, blocks = 0, all;
        bool fresh = false;
        if (k < columns) {
            int hi = B;                                                  // pre[b] <= k < pre[hi]
            while (hi - b > 1) {
                const int mid = (b + hi) >> 1;
                if (pre[mid] <= k) b = mid;
                else hi = mid;
            }
            c = first[b] + k - pre[b];
            page = p.table[b * bt.table_ld + c];
            if (!in_pool(page, n_pages)) page = -1;
            fresh = page < 0 || p.refs[page] > 1;
            if (fresh && page >= 0 && k == pre[b]) {                     // (older tokens lie in front of the first new one only)
                int t0;
                const int older = (int)(max((int64_t)bt.kv_len[b] - paged_rows(bt, b, &t0), (int64_t)0) - ((int64_t)c << log2_page));
                blocks = (older + kPagedBlock - 1) / kPagedBlock;
            }
        }
        const int at = needs + plan_scan((int)fresh, &all, sums);
        if (fresh && at < n_pages) p.need[at] = make_int4(b, c, page, blocks);
        needs += all;
    }
    if (needs == 0) {                                                    // (a generated token in four of a page's places, say)
        if (tid == 0) { *p.missing = 0; *p.n_copies = 0; }
        return;
    }
    // ---- the lowest free pages, in order: each warp counts those of its share, then writes down as many as there are needs
    int lo, hi, n_free = 0, all_free;
    plan_share(n_pages, &lo, &hi);
#pragma unroll 4
    for (int base = lo; base < hi; base += 128) {
        const uint32_t live = plan_live(p.refs, base, hi);
        n_free += __popc(~live & live >> 8 & 15u);
    }
    int before = plan_scan(n_free, &all_free, sums);
    before = __shfl_sync(0xffffffffu, before, 0);                        // (of the warp)
    if (needs > all_free) {
        if (tid == 0) { *p.missing = needs - all_free; *p.n_copies = 0; }
        return;                                                          // (nothing has been changed)
    }
#pragma unroll 4
    for (int base = lo; base < hi && before < needs; base += 128) {
        const uint32_t live = plan_live(p.refs, base, hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool is_free = (~live & live >> 8) >> k & 1;
            const uint32_t mask = __ballot_sync(0xffffffffu, is_free);
            const int at = before + __popc(mask & ((1u << lane) - 1));
            if (is_free && at < needs) p.free_list[at] = base + 32 * k + lane;
            before += __popc(mask);
        }
    }
    __syncthreads();
    for (int j = tid; j < needs; j += kPlanThreads) {
        const int4 n = p.need[j];
        const int page = p.free_list[j];
        p.table[n.x * bt.table_ld + n.y] = page;
        p.refs[page] = 1;
        if (n.z < 0) continue;
        atomicSub(p.refs + n.z, 1);
        if (n.w > 0) p.copies[atomicAdd(&copied, 1)] = make_int4(n.z, page, n.w, 0);
    }
    __syncthreads();
    if (tid == 0) { *p.missing = 0; *p.n_copies = copied; }
}

struct PagedCompactParams {
    int32_t* table;
    int32_t* refs;
    int32_t* moved;              // [n_pages] where a page is now, -1: it was free
    int32_t* movers;             // the workspace, n_pages entries each: the live pages by their rank, the free places
    int32_t* holes;
    int4* copies;
    int32_t* n_copies;
    int8_t* bounds;              // may be null, with scales
    float* scales;
    int64_t table_ld;
    int32_t B, width, n_pages, h_kv, d;
};

// With n live pages, those numbered n and up move to the free places below n, both in order (as many of the one as of the other).
__global__ void __launch_bounds__(kPlanThreads) paged_compact_kernel(const PagedCompactParams p)
{
    __shared__ int sums[kPlanWarps];
    const int tid = threadIdx.x, lane = tid & 31, n_pages = p.n_pages;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int lo, hi, count = 0, n_live;
    plan_share(n_pages, &lo, &hi);
#pragma unroll 4
    for (int base = lo; base < hi; base += 128) count += __popc(plan_live(p.refs, base, hi) & 15u);
    int rank = plan_scan(count, &n_live, sums), n_holes = 0;
    rank = __shfl_sync(0xffffffffu, rank, 0);                            // live pages before the warp's share
#pragma unroll 4
    for (int base = lo; base < hi; base += 128) {
        const uint32_t live = plan_live(p.refs, base, hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int page = base + 32 * k + lane;
            const bool is_live = live >> k & 1;
            const uint32_t mask = __ballot_sync(0xffffffffu, is_live);
            const int mine = rank + __popc(mask & ((1u << lane) - 1));
            rank += __popc(mask);
            if (page >= hi) continue;
            if (is_live && page >= n_live) p.movers[mine] = page;
            else p.moved[page] = is_live ? page : -1;
            if (!is_live && page < n_live) { p.holes[page - mine] = page; ++n_holes; }
        }
    }
    int all_holes;
    plan_scan(n_holes, &all_holes, sums);
    __syncthreads();
    for (int j = tid; j < all_holes; j += kPlanThreads) {
        const int from = p.movers[n_live - all_holes + j], to = p.holes[j];
        p.moved[from] = to;
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
        p.copies[j] = make_int4(from, to, 0, 0);                         // (whole pages)
    }
    if (tid == 0) *p.n_copies = all_holes;
}

struct PagedCopyParams {
    uint8_t* pool;
    const int4* copies;
    const int32_t* n_copies;
    int32_t runs, run_bytes, block_bytes;                                // of a page; block_bytes: of a block, 0 where runs are copied whole
    PagedCompactParams compact;                                          // table null: pages only
};
constexpr int kCopyThreads = 256, kCopyLoads = 4, kCopyPiece = kCopyThreads * kCopyLoads * 16;
static_assert((int64_t)paged_block_bytes(256) * 64 * 1024 <= INT32_MAX - kCopyPiece, "a page of 1024 heads and 1024 tokens is numbered in 32 bits");

// Pages from place to place, a piece of a run of bytes (a page; of a head, where not all of its blocks are wanted) per CTA and turn, with all of a thread's loads in flight.  No place is copied to
// that is copied from: a live page is the one, a free one the other.  Bound: HBM (5000 pages of 74 KB, three times L2 read and written, moved in 121 us, 6.1 TB/s
// or 0.93 of the copy rate; 1000 of them in 22.5, when 46 of the 74 MB written still lie in L2).
__global__ void __launch_bounds__(kCopyThreads) paged_copy_kernel(const PagedCopyParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int n = *p.n_copies, per_run = (p.run_bytes + kCopyPiece - 1) / kCopyPiece, per_page = p.runs * per_run;
    const int64_t page_bytes = (int64_t)p.runs * p.run_bytes;
    for (int64_t item = blockIdx.x; item < (int64_t)n * per_page; item += gridDim.x) {
        const int4 c = p.copies[item / per_page];
        const int in_page = (int)(item % per_page), run = in_page / per_run;
        const int bytes = p.block_bytes ? c.z * p.block_bytes : p.run_bytes, at = (in_page - run * per_run) * kCopyPiece + threadIdx.x * 16;
        const uint8_t* from = p.pool + c.x * page_bytes + (int64_t)run * p.run_bytes;
        uint8_t* to = p.pool + c.y * page_bytes + (int64_t)run * p.run_bytes;
        uint4 u[kCopyLoads];
#pragma unroll
        for (int k = 0; k < kCopyLoads; ++k)
            if (at + k * kCopyThreads * 16 < bytes) u[k] = *reinterpret_cast<const uint4*>(from + at + k * kCopyThreads * 16);
#pragma unroll
        for (int k = 0; k < kCopyLoads; ++k)
            if (at + k * kCopyThreads * 16 < bytes) *reinterpret_cast<uint4*>(to + at + k * kCopyThreads * 16) = u[k];
    }
    const PagedCompactParams& m = p.compact;
    const int64_t t = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x, threads = (int64_t)gridDim.x * kCopyThreads;
    if (m.bounds) {
        const int row = m.h_kv * m.d / 8;                                // 16 bytes each
        for (int64_t e = t; e < (int64_t)n * row; e += threads) {
            const int4 c = p.copies[e / row];
            reinterpret_cast<uint4*>(m.bounds)[(int64_t)c.y * row + e % row] = reinterpret_cast<const uint4*>(m.bounds)[(int64_t)c.x * row + e % row];
        }
        for (int64_t e = t; e < (int64_t)n * m.h_kv; e += threads) {
            const int4 c = p.copies[e / m.h_kv];
            m.scales[(int64_t)c.y * m.h_kv + e % m.h_kv] = m.scales[(int64_t)c.x * m.h_kv + e % m.h_kv];
        }
    }
    if (m.table)
        for (int64_t e = t; e < (int64_t)m.B * m.width; e += threads) {
            int32_t* entry = m.table + e / m.width * m.table_ld + e % m.width;
            if (in_pool(*entry, m.n_pages)) *entry = m.moved[*entry];
        }
}

}  // namespace ql
