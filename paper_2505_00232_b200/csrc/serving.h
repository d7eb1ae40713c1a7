// What the units of the paged cache's calls share on the host: the handle, the checks of a batch, the way a launch ends (serving.cu, pages.cu, contexts.cu).
#pragma once
#include <cuda_runtime.h>

#include <stdint.h>

#include "host.h"
#include "paged.cuh"

struct qlinear_paged_s {
    // Immutable after qlinear_paged_create.
    qlinear_paged_desc d;
    uint8_t* pool;
    int device, log2_blocks;
    int32_t two_ctas_upto;                                               // sequences of an attention call with few rows up to which two CTAs fit on an SM
    ql::SharedState shared;
    bool pdl;
};

namespace ql {

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Bytes of a page; 0 for a descriptor that is not supported.
inline size_t page_bytes(const qlinear_paged_desc* d)
{
    if (!d || d->n_pages < 1 || d->h_kv < 1 || d->h_kv > 1024) return 0;
    if (d->d_h != 64 && d->d_h != 128 && d->d_h != 256) return 0;
    if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1))) return 0;
    if ((int64_t)d->n_pages * d->page_size > INT32_MAX) return 0;
    return (size_t)d->h_kv * (d->page_size / kPagedBlock) * paged_block_bytes(d->d_h);
}

// The batch of a call; false for bad arguments.
inline bool batch_of(qlinear_paged_t h, const int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T, PagedBatch* b)
{
    if (!h || B < 0 || T < 0 || B > QL_PAGED_MAX_SEQUENCES || table_width < 0 || table_ld < table_width) return false;
    if (B > 0 && (!kv_len || !q_start || (!table && table_width > 0))) return false;
    if (!aligned(table, 4) || !aligned(kv_len, 4) || !aligned(q_start, 4)) return false;
    b->pool = h->pool;
    b->table = table;
    b->kv_len = kv_len;
    b->q_start = q_start;
    b->B = B; b->T = T; b->table_width = table_width; b->n_pages = h->d.n_pages; b->log2_blocks = h->log2_blocks; b->h_kv = h->d.h_kv;
    b->table_ld = table_ld;
    return true;
}
inline bool rows_ok(const void* p, int64_t ld, int64_t width) { return p && aligned(p, 16) && ld >= width && ld % 8 == 0; }
inline bool timed_out(qlinear_paged_t h) { return *h->shared.status_host != 0; }
inline unsigned pieces(int64_t n, int64_t size) { return (unsigned)((n + size - 1) / size); }   // (n up to 2^31 - 1)
inline ql_status launched(cudaError_t e)
{
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess ? QL_OK : QL_ERR_CUDA;
}

// The words of the bounded waits of contexts.cu on a device, tied to the device's pinned one (as serving.cu ties its own).
cudaError_t link_contexts(unsigned int* word);

}  // namespace ql
