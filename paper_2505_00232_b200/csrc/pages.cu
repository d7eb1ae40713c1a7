// C-ABI of the calls on the paged cache's pages: forked, released, reserved and compacted page tables, the summaries of pages, and the choice of pages for a query.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdlib>

#include "bounds.cuh"
#include "pages.cuh"
#include "serving.h"

using namespace ql;

namespace {

// A page table that a call may write; false for bad arguments.
bool table_ok(qlinear_paged_t h, const int32_t* table, int64_t ld, int32_t width, int32_t rows)
{
    return h && rows >= 0 && width >= 0 && ld >= width && aligned(table, 4) && (table || rows == 0 || width == 0);
}
// Whether two page tables of the same width have no entry in common: rows between or beside each other's do not.
bool apart(const int32_t* a, int64_t a_ld, int64_t a_rows, const int32_t* b, int64_t b_ld, int64_t b_rows, int64_t width)
{
    if (a_rows == 0 || b_rows == 0 || width == 0) return true;
    const int64_t first = ((int64_t)reinterpret_cast<uintptr_t>(b) - (int64_t)reinterpret_cast<uintptr_t>(a)) / 4;   // of b's entries, from a's on
    if (first >= (a_rows - 1) * a_ld + width || first + (b_rows - 1) * b_ld + width <= 0) return true;
    for (int64_t j = 0; j < b_rows; ++j) {
        const int64_t at = first + j * b_ld, i = std::min(std::max<int64_t>(at, 0) / a_ld, a_rows - 1);   // row i of a begins at or before it, unless that is row 0
        if (std::abs(at - i * a_ld) < width || (i + 1 < a_rows && std::abs(at - (i + 1) * a_ld) < width)) return false;
    }
    return true;
}
bool workspace_ok(qlinear_paged_t h, const void* p, size_t bytes) { return p && aligned(p, 32) && bytes >= qlinear_paged_pages_workspace(h); }
struct Workspace { int4 *copies, *need; int32_t *one, *two, *n_copies; };
Workspace parts_of(qlinear_paged_t h, void* p)
{
    const size_t n = (size_t)h->d.n_pages;
    int4* at = static_cast<int4*>(p);
    int32_t* ints = reinterpret_cast<int32_t*>(at + 2 * n);
    return {at, at + n, ints, ints + n, ints + 2 * n};
}
unsigned copy_grid(const PagedCopyParams& p, int64_t pages, int sms)
{
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>(8 * sms, pages * p.runs * ((p.run_bytes + kCopyPiece - 1) / kCopyPiece)));
}

}  // namespace

extern "C" ql_status qlinear_paged_fork(qlinear_paged_t h, int32_t* refs, const int32_t* table, int64_t table_ld, int32_t table_width, int32_t B, const int32_t* parents, const int32_t* lengths, int32_t n,
                                        int32_t* children, int64_t children_ld, void* stream)
{
    if (!table_ok(h, table, table_ld, table_width, B) || !table_ok(h, children, children_ld, table_width, n) || n > QL_PAGED_MAX_SEQUENCES || !refs || !aligned(refs, 4)) return QL_ERR_INVALID_ARG;
    if (n > 0 && (!parents || !lengths || !aligned(parents, 4) || !aligned(lengths, 4))) return QL_ERR_INVALID_ARG;
    if (!apart(table, table_ld, B, children, children_ld, n, table_width)) return QL_ERR_INVALID_ARG;
    if (n == 0 || table_width == 0) return QL_OK;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    const PagedForkParams p{table, parents, lengths, children, refs, table_ld, children_ld, B, table_width, h->d.n_pages, h->log2_blocks + 4};
    return launched(launch(paged_fork_kernel, p, dim3(pieces(table_width, 256), n), dim3(256), 0, static_cast<cudaStream_t>(stream), 1, h->pdl));
}

extern "C" ql_status qlinear_paged_release(qlinear_paged_t h, int32_t* refs, int32_t* table, int64_t table_ld, int32_t table_width, int32_t B, const int32_t* rows, const int32_t* keep, int32_t n, void* stream)
{
    if (!table_ok(h, table, table_ld, table_width, B) || n < 0 || n > 65535 || !refs || !aligned(refs, 4)) return QL_ERR_INVALID_ARG;
    if (n > 0 && (!rows || !aligned(rows, 4) || !aligned(keep, 4))) return QL_ERR_INVALID_ARG;
    if (n == 0 || B == 0 || table_width == 0) return QL_OK;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    const PagedReleaseParams p{table, rows, keep, refs, table_ld, B, table_width, h->d.n_pages, h->log2_blocks + 4};
    return launched(launch(paged_release_kernel, p, dim3(pieces(table_width, 256), n), dim3(256), 0, static_cast<cudaStream_t>(stream), 1, h->pdl));
}

extern "C" size_t qlinear_paged_pages_workspace(qlinear_paged_t h) { return h ? (size_t)h->d.n_pages * 40 + 64 : 0; }

extern "C" ql_status qlinear_paged_reserve(qlinear_paged_t h, int32_t* refs, int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T,
                                           int32_t* missing, void* workspace, size_t workspace_bytes, void* stream)
{
    PagedReserveParams p{};
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch) || !refs || !aligned(refs, 4) || !missing || !aligned(missing, 4) || !workspace_ok(h, workspace, workspace_bytes)) return QL_ERR_INVALID_ARG;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    const Workspace w = parts_of(h, workspace);
    p.table = table; p.refs = refs; p.missing = missing;
    p.need = w.need; p.free_list = w.one; p.copies = w.copies; p.n_copies = w.n_copies;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch(paged_reserve_kernel, p, dim3(1), dim3(kPlanThreads), (2 * B + 1) * 4, st, 1, h->pdl);
    if (e != cudaSuccess || B == 0 || T == 0) return launched(e);
    const int block = paged_block_bytes(h->d.d_h);
    PagedCopyParams c{h->pool, w.copies, w.n_copies, h->d.h_kv, block << h->log2_blocks, block, {}};
    return launched(launch(paged_copy_kernel, c, dim3(copy_grid(c, B, h->shared.sms)), dim3(kCopyThreads), 0, st, 1, h->pdl));   // (a sequence's older tokens end in one page)
}

extern "C" ql_status qlinear_paged_compact(qlinear_paged_t h, int32_t* refs, int32_t* table, int64_t table_ld, int32_t table_width, int32_t B, void* bounds, float* scales, int32_t* moved,
                                           void* workspace, size_t workspace_bytes, void* stream)
{
    if (!table_ok(h, table, table_ld, table_width, B) || !refs || !aligned(refs, 4) || !moved || !aligned(moved, 4) || !workspace_ok(h, workspace, workspace_bytes)) return QL_ERR_INVALID_ARG;
    if ((bounds == nullptr) != (scales == nullptr) || !aligned(bounds, 16) || !aligned(scales, 4)) return QL_ERR_INVALID_ARG;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    const Workspace w = parts_of(h, workspace);
    const PagedCompactParams p{B > 0 && table_width > 0 ? table : nullptr, refs, moved, w.one, w.two, w.copies, w.n_copies, static_cast<int8_t*>(bounds), scales, table_ld, B, table_width, h->d.n_pages,
                               h->d.h_kv, h->d.d_h};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch(paged_compact_kernel, p, dim3(1), dim3(kPlanThreads), 0, st, 1, h->pdl);
    if (e != cudaSuccess) return launched(e);
    const PagedCopyParams c{h->pool, w.copies, w.n_copies, 1, (int)page_bytes(&h->d), 0, p};
    return launched(launch(paged_copy_kernel, c, dim3(8 * h->shared.sms), dim3(kCopyThreads), 0, st, 1, h->pdl));
}

extern "C" ql_status qlinear_paged_summarise(qlinear_paged_t h, const int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T,
                                             void* bounds, float* scales, void* stream)
{
    PagedBoundsParams p{};
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch) || !bounds || !scales || !aligned(bounds, 16) || !aligned(scales, 4)) return QL_ERR_INVALID_ARG;
    if (B == 0 || T == 0 || table_width == 0) return QL_OK;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    p.bounds = static_cast<int8_t*>(bounds);
    p.scales = scales;
    // T rows of B sequences lie in T / page_size + 2 B pages at most
    const int64_t pages = std::min<int64_t>(((int64_t)T >> (h->log2_blocks + 4)) + 2ll * B, T);
    const unsigned grid = (unsigned)std::min<int64_t>(pages, (h->d.d_h == 256 ? 2ll : 4ll) * h->shared.sms);
    const auto kernel = h->d.d_h == 64 ? paged_bounds_kernel<64> : h->d.d_h == 128 ? paged_bounds_kernel<128> : paged_bounds_kernel<256>;
    return launched(launch(kernel, p, dim3(grid), dim3(kBoundsThreads), (3 * B + 1) * 4, static_cast<cudaStream_t>(stream), 1, h->pdl));
}

namespace {
template <int D>
cudaError_t launch_select(const PagedSelectParams& p, dim3 grid, int cluster, int device, cudaStream_t st, bool pdl)
{
    static std::atomic<bool> flags[64];
    if (!flags[device].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(paged_select_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, std::max(kSelectMostColumns / 8, kSelectGathered) * 4);
        if (e != cudaSuccess) return e;
        flags[device].store(true, std::memory_order_release);
    }
    return launch(paged_select_kernel<D>, p, grid, dim3(kSelectThreads), (p.gathered ? p.batch.table_width : p.share) * 4, st, cluster, pdl);
}
}  // namespace

extern "C" ql_status qlinear_paged_select(qlinear_paged_t h, const void* q, int64_t q_ld, int32_t h_q, const void* bounds, const float* scales,
                                          const int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T,
                                          int32_t budget, int32_t first, int32_t recent, int32_t* pages, void* stream)
{
    PagedSelectParams p{};
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch) || table_width > kSelectMostColumns) return QL_ERR_INVALID_ARG;
    if (h_q < 1 || h_q > 65536 || h_q % h->d.h_kv || budget < 1 || first < 0 || recent < 0 || (int64_t)first + recent > budget) return QL_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return QL_OK;
    if (!rows_ok(q, q_ld, (int64_t)h_q * h->d.d_h) || !bounds || !scales || !aligned(bounds, 16) || !aligned(scales, 4) || !pages || !aligned(pages, 4)) return QL_ERR_INVALID_ARG;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    p.q = static_cast<const __half*>(q); p.q_ld = q_ld;
    p.bounds = static_cast<const int8_t*>(bounds); p.scales = scales; p.pages = pages;
    p.group = h_q / h->d.h_kv; p.budget = budget; p.first = first; p.recent = recent;
    // CTAs of a row and KV head: more while they would not fill the SMs twice and have 64 columns left each, and as many as hold the keys (us, clusters of 1, 2, 4, 8: one row of 8 heads and 2048 pages 23.1, 15.6, 11.9,
    // 10.3; 32 ragged rows of up to 1024 pages 16.5, 14.9, 17.2, 24.2; 16 rows of 4 heads of 256 and 1000 pages 22.2, 15.9, 13.4, 14.3)
    int cluster = 1;
    while (cluster < 8 && (int64_t)T * h->d.h_kv * cluster <= 2 * h->shared.sms && table_width / (2 * cluster) >= 64) cluster *= 2;
    p.gathered = table_width <= kSelectGathered;
    while (!p.gathered && (table_width + cluster - 1) / cluster > kSelectMostColumns / 8) cluster *= 2;
    p.share = std::max((table_width + cluster - 1) / cluster, 1);
    if ((int64_t)T * cluster > INT32_MAX) return QL_ERR_INVALID_ARG;
    const auto go = h->d.d_h == 64 ? launch_select<64> : h->d.d_h == 128 ? launch_select<128> : launch_select<256>;
    return launched(go(p, dim3((unsigned)T * cluster, h->d.h_kv), cluster, h->device, static_cast<cudaStream_t>(stream), h->pdl));
}
