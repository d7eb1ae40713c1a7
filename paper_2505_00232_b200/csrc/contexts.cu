// C-ABI of the attention calls over shared and sparse contexts of the paged cache: a shared beginning once for all rows of a group, and pages listed for a row.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>

#include "host.h"

namespace ql {
// This unit's words of the bounded waits (sm100_ptx.cuh): the host reads the pinned one, which the whole device shares.
static __device__ unsigned int g_device_flag[2];
static __device__ unsigned int* g_status_host;
}  // namespace ql

#include "paged_attention.cuh"
#include "paged_shared.cuh"
#include "paged_tiles.cuh"
#include "serving.h"

using namespace ql;

cudaError_t ql::link_contexts(unsigned int* word) { return cudaMemcpyToSymbol(g_status_host, &word, sizeof(word)); }

namespace {

template <int D> constexpr int few_smem(int32_t n) { return AttnRing<D>::kBytes + (n + 1) * 4; }
template <int D> constexpr int tiles_smem(int32_t n) { return 1024 + TileShape<D>::kOffPre + (n + 1) * 4; }

// Scores' parameters of a call; false for bad arguments.
bool scores_of(float scale, float softcap, PagedAttnParams* p)
{
    if (!(std::fabs(scale) <= kMostScale) || !(softcap >= 0.f) || !std::isfinite(softcap)) return false;
    p->scale = scale;
    // (a cap below makes all scores one to 30 digits, a cap above leaves them what they are)
    p->softcap = softcap > 0.f ? std::min(std::max(softcap, 1e-30f * std::max(std::fabs(scale), 1.f)), 1e38f) : 0.f;
    return true;
}

template <int D, AttnCap CAP, AttnKind KIND>
cudaError_t launch_few_as(const PagedAttnParams& p, int32_t n, int device, cudaStream_t st, bool pdl)
{
    static std::atomic<bool> flags[64];
    if (!flags[device].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(paged_attention_kernel<D, CAP, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, few_smem<D>(QL_PAGED_MAX_SEQUENCES));
        if (e != cudaSuccess) return e;
        flags[device].store(true, std::memory_order_release);
    }
    return launch(paged_attention_kernel<D, CAP, KIND>, p, dim3(p.grid), dim3(kAttnWarps * 32), few_smem<D>(n), st, 1, pdl);
}
template <int D, AttnKind KIND>
cudaError_t launch_few(const PagedAttnParams& p, int32_t n, int device, cudaStream_t st, bool pdl)
{
    if (!(p.softcap > 0.f)) return launch_few_as<D, kCapNone, KIND>(p, n, device, st, pdl);
    return p.softcap <= kMostPlainCap ? launch_few_as<D, kCapPlain, KIND>(p, n, device, st, pdl) : launch_few_as<D, kCapHigh, KIND>(p, n, device, st, pdl);
}
template <int D, AttnCap CAP>
cudaError_t launch_tiles_as(const PagedAttnParams& p, int32_t n, int device, cudaStream_t st, bool pdl)
{
    static std::atomic<bool> flags[64];
    if (!flags[device].load(std::memory_order_acquire)) {
        cudaError_t e = cudaFuncSetAttribute(paged_tiles_kernel<D, CAP, kAttnShared>, cudaFuncAttributeMaxDynamicSharedMemorySize, tiles_smem<D>(QL_PAGED_MAX_SEQUENCES));
        cudaFuncAttributes at;
        if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, paged_tiles_kernel<D, CAP, kAttnShared>);
        if (e != cudaSuccess) return e;
        if (at.numRegs < kTileRegisters) return cudaErrorInvalidConfiguration;   // (the roles' shares come from what the block was launched with: they would be waited for)
        flags[device].store(true, std::memory_order_release);
    }
    return launch(paged_tiles_kernel<D, CAP, kAttnShared>, p, dim3(p.grid), dim3(kTileThreads), tiles_smem<D>(n), st, 1, pdl);
}
template <int D>
cudaError_t launch_tiles(const PagedAttnParams& p, int32_t n, int device, cudaStream_t st, bool pdl)
{
    if (!(p.softcap > 0.f)) return launch_tiles_as<D, kCapNone>(p, n, device, st, pdl);
    return p.softcap <= kMostPlainCap ? launch_tiles_as<D, kCapPlain>(p, n, device, st, pdl) : launch_tiles_as<D, kCapHigh>(p, n, device, st, pdl);
}

int32_t few_ctas(qlinear_paged_t h, int32_t n) { return (n > h->two_ctas_upto ? 1 : 2) * h->shared.sms; }   // (those that run at once; the kinds differ in a few bytes of shared memory)
size_t few_partial(qlinear_paged_t h) { return (size_t)4 * h->shared.sms * kAttnCols * (h->d.d_h + 2) * sizeof(float); }

}  // namespace

// ---------------------------------------------------------------------------------------------------- pages listed for a row
extern "C" size_t qlinear_paged_attention_selected_workspace(qlinear_paged_t h, int32_t h_q)
{
    return h && h_q >= 1 && h_q <= 65536 && h_q % h->d.h_kv == 0 ? few_partial(h) + (size_t)2 * h->shared.sms * sizeof(int4) : 0;
}

namespace {
template <int D>
cudaError_t launch_selected(const PagedAttnParams& p, int device, cudaStream_t st, bool pdl)
{
    const cudaError_t e = launch_few<D, kAttnListed>(p, p.batch.B, device, st, pdl);
    if (e != cudaSuccess) return e;
    return launch(paged_combine_kernel<D, kAttnCols, 1, 4, kAttnListed>, p, dim3(p.grid, (std::min(kAttnCols, p.group) + 1) / 2), dim3(256), 0, st, 1, pdl);
}
}  // namespace

extern "C" ql_status qlinear_paged_attention_selected(qlinear_paged_t h, const void* q, int64_t q_ld, void* out, int64_t out_ld, int32_t h_q, const int32_t* pages, int32_t budget,
                                                      const int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T,
                                                      float scale, float softcap, void* workspace, size_t workspace_bytes, void* stream)
{
    PagedAttnParams p{};
    const size_t bytes = qlinear_paged_attention_selected_workspace(h, h_q);
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch) || bytes == 0 || budget < 0 || !scores_of(scale, softcap, &p)) return QL_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return QL_OK;
    const int32_t d = h->d.d_h;
    p.group = h_q / h->d.h_kv;
    p.row_blocks = (p.group + kAttnCols - 1) / kAttnCols;
    // the kernel numbers the blocks of all rows in 32 bits
    if ((__int128)T * (((int64_t)budget << h->log2_blocks) + kAttnOverhead + 1) * p.row_blocks > INT32_MAX) return QL_ERR_INVALID_ARG;
    if (!rows_ok(q, q_ld, (int64_t)h_q * d) || !rows_ok(out, out_ld, (int64_t)h_q * d) || q == out || !aligned(pages, 4) || (!pages && budget > 0)) return QL_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 32) || workspace_bytes < bytes) return QL_ERR_INVALID_ARG;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    p.q = static_cast<const __half*>(q); p.out = static_cast<__half*>(out);
    p.q_ld = q_ld; p.out_ld = out_ld;
    p.h_q = h_q; p.max_q = INT32_MAX; p.pages = pages; p.budget = budget;
    p.partial = static_cast<float*>(workspace);
    p.split = reinterpret_cast<int4*>(static_cast<char*>(workspace) + few_partial(h));
    p.grid = few_ctas(h, B);
    const auto go = d == 64 ? launch_selected<64> : d == 128 ? launch_selected<128> : launch_selected<256>;
    return launched(go(p, h->device, static_cast<cudaStream_t>(stream), h->pdl));
}

// ---------------------------------------------------------------------------------------------------- a shared beginning
namespace {

struct SharedPlan {
    bool alone;                                                          // the call is one of qlinear_paged_attention
    bool prefix_tiles, own_tiles;
    int32_t group, tile_rows;
    size_t own_at, rows_at, ml_at, stretches_at, lengths_at, row_of_at, spans_at, bytes;
};
// Which kernels take it: by estimates of the three ways' times, with the table's columns for the lengths and three quarters of them for the beginnings.  A launch over stretches has a fixed part (plan, ramps, join; the tiles a pipeline of their
// own), few rows cost by their blocks of 16 tokens and 8 rows, tiles by their steps of 64 tokens.  us, plain, few rows and tiles, 8 KV heads of 128 and 4 queries each: 4 sequences over 1024 tokens 11.5, 14.9, 30.9; 16 over 2048 19.8, 20.5, 33.1;
// 8 over 16384 41.0, 30.4, 43.4; 16 over 16384 71.5, 47.3, 44.5; two groups of 32 over 16384 259, 149, 75; 16 drafted tokens each, 4 over 16384 81.9, -, 43.6.  4 of 256 and 2: 4 over 16384 25.6, 18.4, 37.7; two groups of 32 257, 87, 61.
// 2 of 64 and 7: 8 over 16384 15.4, 18.4, 32.2; two groups of 32 50, 51, 39.  What the estimate does not know is how long the beginnings are: 64 sequences of 2000 tokens of their own over 512 take 58.6 by its choice and 54.5 plain.
// Nor how long the sequences are, where the table is wider: with 131072 tokens of columns and three quarters of every sequence shared, by its choice and plain, 8 KV heads and 4 queries each: 4 of 1000 16.5, 12.7; 32 of 1000 40.7, 22.6; 32 of 8000
// 59.5, 73.8; 32 of 30000 123, 236.  1 of 128 and 12: 32 of 1000 40.9, 14.7; 32 of 8000 45.1, 28.7; 32 of 30000 59.9, 67.7.
void shared_route(qlinear_paged_t h, int32_t B, int32_t T, int32_t max_q, int32_t n_groups, int32_t table_width, SharedPlan* a)
{
    const int32_t d = h->d.d_h, V = n_groups + B, choice = paged_shared_choice();
    const int64_t held = std::min((int64_t)table_width * h->d.page_size, (int64_t)INT32_MAX), all_rows = (int64_t)T * a->group;
    a->alone = n_groups == 0 || all_rows >= 1 << 30 || choice == 0;
    // (the kernels number the steps of a KV head's segments in 32 bits)
    const __int128 few_blocks = (__int128)(all_rows / kAttnCols + V) * (held / kPagedBlock + 1 + kAttnOverhead), tile_steps = (__int128)(all_rows / a->tile_rows + 2 * V) * (held / 64 + 1 + kTileOverhead);
    if (few_blocks + tile_steps > INT32_MAX) a->alone = true;
    if (a->alone) return;
    const int64_t group_rows = (all_rows + n_groups - 1) / n_groups, rows = (int64_t)max_q * a->group;
    const auto pieces_of = [](int64_t n, int64_t size) { return (double)((n + size - 1) / size); };
    const double per_block = (d == 64 ? 0.085 : d == 128 ? 0.15 : 0.14) * h->d.h_kv * held / kPagedBlock / few_ctas(h, V), per_step = (d == 256 ? 1.4 : 1.1) * h->d.h_kv * held / 64 / h->shared.sms;
    const double beginning = 0.75, each = a->own_tiles ? per_step * B * pieces_of(rows, a->tile_rows) : per_block * B * pieces_of(rows, kAttnCols);   // (of every sequence's whole length)
    const double plain = (a->own_tiles ? 23 : 9.5) + each;
    const double few = a->own_tiles ? INFINITY : 13.5 + (1 - beginning) * each + beginning * per_block * n_groups * pieces_of(group_rows, kAttnCols);
    const double tiles = 28 + (1 - beginning) * each + beginning * per_step * n_groups * pieces_of(group_rows, a->tile_rows);
    a->prefix_tiles = choice == 2 || a->own_tiles || (choice != 1 && tiles < few);
    a->alone = choice < 0 && plain <= std::min(few, tiles);
}

// The launches of a call, from what the host knows of it; false for bad arguments.
bool shared_plan(qlinear_paged_t h, int32_t h_q, int32_t table_width, int32_t B, int32_t T, int32_t max_q, int32_t n_groups, SharedPlan* a)
{
    if (!h || h_q < 1 || h_q > 65536 || h_q % h->d.h_kv || table_width < 0 || B < 0 || T < 0 || n_groups < 0 || max_q < 0 || (int64_t)n_groups + B > QL_PAGED_MAX_SEQUENCES) return false;
    const int32_t d = h->d.d_h;
    a->group = h_q / h->d.h_kv;
    a->tile_rows = d == 256 ? TileShape<256>::kRows : TileShape<128>::kRows;
    a->own_tiles = (int64_t)max_q * a->group > attn_max_rows(d);
    a->bytes = qlinear_paged_attention_workspace(h, h_q, B, max_q);
    shared_route(h, B, T, max_q, n_groups, table_width, a);
    if (a->alone) return a->bytes > 0;
    const auto up = [](size_t n) { return (n + 31) / 32 * 32; };
    const size_t few = up(few_partial(h)), tiles = up((size_t)2 * h->shared.sms * a->tile_rows * (d + 2) * sizeof(float)), cells = (size_t)2 * T * h_q, V = (size_t)n_groups + B;
    a->own_at = a->prefix_tiles ? tiles : 0;                             // (where it is a launch of its own)
    a->rows_at = a->own_at + (a->own_tiles ? 0 : few);
    a->ml_at = a->rows_at + up(cells * d * sizeof(float));
    a->stretches_at = a->ml_at + up(cells * sizeof(float2));
    a->lengths_at = a->stretches_at + up(V * sizeof(AttnStretch));
    a->row_of_at = a->lengths_at + up((V + 1) * 4);
    a->spans_at = a->row_of_at + up((size_t)T * sizeof(int2));
    a->bytes = a->spans_at + 32;
    return true;
}
template <int D>
cudaError_t launch_join(const SharedJoinParams& j, int sms, cudaStream_t st, bool pdl)
{
    // a row's parts are up to one per CTA: warps for them while the SMs have room, 32 each (us, 1, 2, 4, 8 warps a row: 2048 rows of 128 with 20 parts 10.5, 7.1, 10.2, 13.2; 1536 of 256 with 13 10.9, 9.1, 8.5, 11.6; 48 rows
    // with 131 parts: the whole call 76 with one, 33 with eight and parts of 8 steps at least)
    const int64_t rows = (int64_t)j.T * j.h_q, room = 32ll * sms;
    const auto go = [&](auto kernel, int w) { return launch(kernel, j, dim3(j.T, j.h_kv, (j.group + 8 / w - 1) / (8 / w)), dim3(256), 0, st, 1, pdl); };
    if (rows * 8 <= room || j.group <= 1) return go(paged_shared_join_kernel<D, 8>, 8);
    if (rows * 4 <= room || j.group <= 2) return go(paged_shared_join_kernel<D, 4>, 4);
    if (rows * 2 <= room || j.group <= 4) return go(paged_shared_join_kernel<D, 2>, 2);
    return go(paged_shared_join_kernel<D, 1>, 1);
}
template <int D>
cudaError_t launch_shared(const SharedPlanParams& plan, PagedAttnParams p, const SharedJoinParams& j, qlinear_paged_t h, cudaStream_t st)
{
    cudaError_t e = launch(paged_shared_plan_kernel, plan, dim3(1), dim3(kSharedThreads), 0, st, 1, h->pdl);
    const auto go = [&](const SharedLaunch& at) {
        if (e != cudaSuccess) return;
        p.partial = const_cast<float*>(at.partial);
        p.v0 = at.v0; p.v1 = at.v1; p.grid = at.grid;
        e = at.tiles ? launch_tiles<D>(p, at.v1 - at.v0, h->device, st, h->pdl) : launch_few<D, kAttnShared>(p, at.v1 - at.v0, h->device, st, h->pdl);
    };
    go(j.prefix);
    if (j.own.v0 != j.prefix.v0) go(j.own);
    return e != cudaSuccess ? e : launch_join<D>(j, h->shared.sms, st, h->pdl);
}

}  // namespace

extern "C" size_t qlinear_paged_attention_shared_workspace(qlinear_paged_t h, int32_t h_q, int32_t table_width, int32_t B, int32_t T, int32_t max_q, int32_t n_groups)
{
    SharedPlan a;
    return shared_plan(h, h_q, table_width, B, T, max_q, n_groups, &a) ? a.bytes : 0;
}

extern "C" ql_status qlinear_paged_attention_shared(qlinear_paged_t h, const void* q, int64_t q_ld, void* out, int64_t out_ld, int32_t h_q,
                                                    const int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T, int32_t max_q,
                                                    const int32_t* group_start, const int32_t* prefix_len, int32_t n_groups, float scale, float softcap,
                                                    void* workspace, size_t workspace_bytes, void* stream)
{
    PagedAttnParams p{};
    SharedPlan a;
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch) || !shared_plan(h, h_q, table_width, B, T, max_q, n_groups, &a) || !scores_of(scale, softcap, &p)) return QL_ERR_INVALID_ARG;
    if (n_groups > 0 && (!group_start || !prefix_len || !aligned(group_start, 4) || !aligned(prefix_len, 4))) return QL_ERR_INVALID_ARG;
    if (a.alone) return qlinear_paged_attention(h, q, q_ld, out, out_ld, h_q, table, table_ld, table_width, kv_len, q_start, B, T, max_q, scale, softcap, 0, workspace, workspace_bytes, stream);
    if (B == 0 || T == 0 || max_q == 0) return QL_OK;
    const int32_t d = h->d.d_h, V = n_groups + B;
    if (!rows_ok(q, q_ld, (int64_t)h_q * d) || !rows_ok(out, out_ld, (int64_t)h_q * d) || q == out) return QL_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 32) || workspace_bytes < a.bytes) return QL_ERR_INVALID_ARG;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    char* w = static_cast<char*>(workspace);
    const int32_t few = few_ctas(h, V), sms = h->shared.sms;
    const bool one = a.prefix_tiles == a.own_tiles;                      // one launch for both
    const SharedLaunch prefix{reinterpret_cast<const float*>(w), 0, one ? V : n_groups, a.prefix_tiles ? sms : few, a.prefix_tiles};
    const SharedLaunch own = one ? prefix : SharedLaunch{reinterpret_cast<const float*>(w + a.own_at), n_groups, V, a.own_tiles ? sms : few, a.own_tiles};
    int64_t* spans = reinterpret_cast<int64_t*>(w + a.spans_at);
    const SharedPlanParams plan{p.batch, group_start, prefix_len, n_groups, a.group, max_q, a.tile_rows, prefix, own, spans, reinterpret_cast<AttnStretch*>(w + a.stretches_at),
                                reinterpret_cast<int32_t*>(w + a.lengths_at), reinterpret_cast<int2*>(w + a.row_of_at)};
    p.q = static_cast<const __half*>(q); p.q_ld = q_ld;
    p.h_q = h_q; p.group = a.group; p.max_q = max_q; p.n_groups = n_groups;
    p.stretches = plan.stretches; p.lengths = plan.lengths;
    p.row_o = reinterpret_cast<float*>(w + a.rows_at); p.row_ml = reinterpret_cast<float2*>(w + a.ml_at);
    const SharedJoinParams j{plan.stretches, plan.lengths, plan.row_of, p.row_o, p.row_ml, static_cast<__half*>(out), out_ld, T, h_q, a.group, h->d.h_kv, a.tile_rows == 128 ? 7 : 8, prefix, own, spans};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto go = d == 64 ? launch_shared<64> : d == 128 ? launch_shared<128> : launch_shared<256>;
    return launched(go(plan, p, j, h, st));
}
