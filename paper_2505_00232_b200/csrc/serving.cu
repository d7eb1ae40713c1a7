// C-ABI of the operators of a serving step around the layers: rotary angle tables, the paged KV cache held in 4 bits (append with the
// rotation, read back, attention), and the adjustment of logits.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <new>

#include "host.h"

namespace ql {
// This unit's words of the bounded waits (sm100_ptx.cuh): the host reads the pinned one, which the whole device shares.
static __device__ unsigned int g_device_flag[2];
static __device__ unsigned int* g_status_host;
}  // namespace ql

#include "logits.cuh"
#include "paged.cuh"
#include "paged_attention.cuh"
#include "paged_tiles.cuh"
#include "rope_tables.cuh"
#include "serving.h"

using namespace ql;

namespace {

// The dynamic shared memory of the kernel of few rows (its plan holds a number per sequence), and up to how many sequences two of its CTAs fit on an SM: at d_h 64 any number, at 128
// about 1660, at 256 none, since its queries lie in shared memory.
template <int D> constexpr int attn_smem(int32_t B) { return AttnRing<D>::kBytes + (B + 1) * 4; }
template <int D>
cudaError_t two_ctas_upto(int device, int32_t* sequences)
{
    int all = 0, reserved = 0, fixed = 0;
    cudaError_t e = cudaDeviceGetAttribute(&all, cudaDevAttrMaxSharedMemoryPerMultiprocessor, device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&reserved, cudaDevAttrReservedSharedMemoryPerBlock, device);
    for (const auto kernel : {paged_attention_kernel<D, kCapNone>, paged_attention_kernel<D, kCapPlain>, paged_attention_kernel<D, kCapHigh>}) {
        cudaFuncAttributes at;
        if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, kernel);
        if (e == cudaSuccess) fixed = std::max(fixed, (int)at.sharedSizeBytes);
    }
    *sequences = (all / 2 / 128 * 128 - reserved - fixed - attn_smem<D>(0)) / 4;   // (shared memory is given out 128 bytes at a time)
    return e;
}

}  // namespace

// ---------------------------------------------------------------------------------------------------- rotary angle tables
extern "C" ql_status qlinear_rope_tables(float* cos_dev, float* sin_dev, int32_t first, int32_t n_pos, int32_t rot, double base, const qlinear_rope_scaling* s, int32_t device, void* stream)
{
    if (n_pos < 0 || first < 0 || (int64_t)first + n_pos > INT32_MAX || rot < 16 || rot % 16 || rot > 2 * kRopeTablesMaxPairs || !(base > 1.0) || !std::isfinite(base) || device < 0) return QL_ERR_INVALID_ARG;
    const int32_t kind = s ? s->kind : QL_ROPE_NONE;
    if (kind < QL_ROPE_NONE || kind > QL_ROPE_YARN) return QL_ERR_INVALID_ARG;
    if (kind != QL_ROPE_NONE && (!(s->factor >= 1.0) || !std::isfinite(s->factor))) return QL_ERR_INVALID_ARG;
    if ((kind == QL_ROPE_LLAMA3 || kind == QL_ROPE_YARN) && (s->original < 1 || !(s->slow > 0.0) || !(s->fast > s->slow) || !std::isfinite(s->fast))) return QL_ERR_INVALID_ARG;
    if (n_pos == 0) return QL_OK;
    if (!cos_dev || !sin_dev || !aligned(cos_dev, 16) || !aligned(sin_dev, 16) || cos_dev == sin_dev) return QL_ERR_INVALID_ARG;
    RopeTablesParams p{};
    p.cos_t = cos_dev; p.sin_t = sin_dev; p.first = first; p.n_pos = n_pos; p.pairs = rot / 2;
    p.magnitude = kind == QL_ROPE_YARN ? (float)(0.1 * std::log(s->factor) + 1.0) : 1.f;
    constexpr double kTwoPi = 6.283185307179586476925286766559;
    if (kind == QL_ROPE_NTK) base *= std::pow(s->factor, rot / (rot - 2.0));
    double low = 0.0, high = 0.0;
    if (kind == QL_ROPE_YARN) {
        const auto pair_of = [&](double turns) { return rot * std::log(s->original / (turns * kTwoPi)) / (2.0 * std::log(base)); };
        low = std::max(std::floor(pair_of(s->fast)), 0.0);
        high = std::min(std::ceil(pair_of(s->slow)), rot - 1.0);
    }
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot);
        if (kind == QL_ROPE_LINEAR) f /= s->factor;
        if (kind == QL_ROPE_LLAMA3) {                                    // by the turns that a pair makes within the original length
            const double keep = std::min(1.0, std::max(0.0, (s->original * f / kTwoPi - s->slow) / (s->fast - s->slow)));
            f = f / s->factor * (1.0 - keep) + f * keep;
        }
        if (kind == QL_ROPE_YARN) {                                      // the same over the pairs' numbers
            const double slowed = std::min(1.0, std::max(0.0, (i - low) / std::max(high - low, 0.001)));
            f = f / s->factor * slowed + f * (1.0 - slowed);
        }
        const double turns = f / kTwoPi;
        p.turns[i] = (uint64_t)std::ldexp(turns - std::floor(turns), 64);   // (below one turn: base > 1)
    }
    int sms;
    const ql_status ready = device_sms(device, &sms);
    if (ready != QL_OK) return ready;
    DeviceGuard guard(device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    const int per_block = 256 / (p.pairs / 4);
    return launched(launch(rope_tables_kernel, p, dim3(std::min(pieces(n_pos, per_block), 8u * sms)), dim3(256), 0, static_cast<cudaStream_t>(stream), 1, pdl_enabled()));
}

// ---------------------------------------------------------------------------------------------------- paged cache
extern "C" size_t qlinear_paged_page_bytes(const qlinear_paged_desc* d) { return page_bytes(d); }

extern "C" ql_status qlinear_paged_create(const qlinear_paged_desc* d, void* pool_dev, int device, qlinear_paged_t* out)
{
    if (!d || !pool_dev || !out) return QL_ERR_INVALID_ARG;
    *out = nullptr;
    if (page_bytes(d) == 0) return QL_ERR_UNSUPPORTED;
    if (!aligned(pool_dev, 256)) return QL_ERR_INVALID_ARG;
    SharedState shared;
    const ql_status st = shared_state(device, &shared);
    if (st != QL_OK) return st;
    {
        // the kernels of this unit and of contexts.cu report an expired wait through the device's pinned word as well
        static std::atomic<bool> linked[64];
        DeviceGuard guard(device);
        if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
        unsigned int* word = nullptr;
        if (!linked[device].load(std::memory_order_acquire)) {
            if (cudaHostGetDevicePointer(reinterpret_cast<void**>(&word), const_cast<unsigned int*>(shared.status_host), 0) != cudaSuccess ||
                cudaMemcpyToSymbol(g_status_host, &word, sizeof(word)) != cudaSuccess || link_contexts(word) != cudaSuccess) { cudaGetLastError(); return QL_ERR_CUDA; }
            linked[device].store(true, std::memory_order_release);
        }
    }
    int32_t upto = 0;
    {
        DeviceGuard guard(device);
        if (!guard.ok || (d->d_h == 64 ? two_ctas_upto<64> : d->d_h == 128 ? two_ctas_upto<128> : two_ctas_upto<256>)(device, &upto) != cudaSuccess) { cudaGetLastError(); return QL_ERR_CUDA; }
    }
    qlinear_paged_s* h = new (std::nothrow) qlinear_paged_s();
    if (!h) return QL_ERR_ALLOC;
    h->d = *d;
    h->pool = static_cast<uint8_t*>(pool_dev);
    h->device = device;
    h->two_ctas_upto = upto;
    for (h->log2_blocks = 0; (kPagedBlock << h->log2_blocks) < d->page_size; ++h->log2_blocks) {}
    h->shared = shared;
    h->pdl = pdl_enabled();
    *out = h;
    return QL_OK;
}

extern "C" ql_status qlinear_paged_destroy(qlinear_paged_t h)
{
    delete h;
    return QL_OK;
}

extern "C" ql_status qlinear_paged_device_status(qlinear_paged_t h, uint32_t* detail) { return h ? device_status(h->device, detail) : QL_ERR_INVALID_ARG; }

extern "C" ql_status qlinear_paged_append(qlinear_paged_t h, const void* q, int64_t q_ld, const void* k, int64_t k_ld, const void* v, int64_t v_ld, void* q_out, int64_t q_out_ld, int32_t h_q,
                                          const int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T,
                                          const float* cos_dev, const float* sin_dev, int32_t n_pos, int32_t rot, int32_t interleaved, void* stream)
{
    PagedAppendParams p{};
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch)) return QL_ERR_INVALID_ARG;
    const int32_t d = h->d.d_h, h_kv = h->d.h_kv;
    if (q_out && !q) return QL_ERR_INVALID_ARG;
    if (q && (h_q < 1 || h_q > 65536)) return QL_ERR_INVALID_ARG;
    if ((cos_dev == nullptr) != (sin_dev == nullptr)) return QL_ERR_INVALID_ARG;
    if (T > 0) {
        if (!rows_ok(k, k_ld, (int64_t)h_kv * d) || !rows_ok(v, v_ld, (int64_t)h_kv * d)) return QL_ERR_INVALID_ARG;
        if (q && (!rows_ok(q, q_ld, (int64_t)h_q * d) || !rows_ok(q_out, q_out_ld, (int64_t)h_q * d) || (q == q_out && q_ld != q_out_ld))) return QL_ERR_INVALID_ARG;
    }
    if (cos_dev && (n_pos < 1 || rot < 16 || rot % 16 || rot > d || !aligned(cos_dev, 16) || !aligned(sin_dev, 16) || (interleaved != 0 && interleaved != 1))) return QL_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return QL_OK;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    p.q = static_cast<const __half*>(q); p.k = static_cast<const __half*>(k); p.v = static_cast<const __half*>(v);
    p.q_out = static_cast<__half*>(q_out);
    p.q_ld = q_ld; p.k_ld = k_ld; p.v_ld = v_ld; p.q_out_ld = q_out_ld;
    p.cos_t = cos_dev; p.sin_t = sin_dev; p.n_pos = cos_dev ? n_pos : 1; p.rot = cos_dev ? rot : 0; p.interleaved = interleaved;
    p.h_q = q ? h_q : 0; p.d = d;
    const int passes = ((p.h_q + 2 * h_kv) * (d / 8) + kPagedThreads - 1) / kPagedThreads, sms = h->shared.sms;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // few rows: the passes over the heads as CTAs of their own; many: several rows to a CTA, which looks its sequences up once
    if (T <= 16 * sms) return launched(launch(paged_append_kernel<1>, p, dim3(T, T <= 2 * sms ? std::min(passes, 64) : 1), dim3(kPagedThreads), 0, st, 1, h->pdl));
    return launched(launch(paged_append_kernel<4>, p, dim3((T + 3) / 4), dim3(kPagedThreads), 0, st, 1, h->pdl));
}

extern "C" ql_status qlinear_paged_read(qlinear_paged_t h, const int32_t* table, int64_t table_ld, int32_t table_width, const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T,
                                        void* k_out, void* v_out, void* stream)
{
    PagedReadParams p{};
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch)) return QL_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return QL_OK;
    if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16) || k_out == v_out) return QL_ERR_INVALID_ARG;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    p.k = static_cast<__half*>(k_out); p.v = static_cast<__half*>(v_out); p.d = h->d.d_h;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // rows in a row of their sequences: by blocks; a token of a sequence or a few, and calls of a few hundred rows, by rows (44 rows of 4 sequences, 8 heads of 128: 3.1 us by rows, 4.0 by blocks; 1400 of 6, 4 heads of 256: 6.7 and 6.0;
    // 9500 of 256: 14.3 and 9.7)
    if (T / 8 >= B && T > 2 * h->shared.sms) {
        const int64_t blocks = (int64_t)T / kPagedBlock + 2 * B;         // (at most)
        const unsigned grid = (unsigned)std::min<int64_t>((blocks * h->d.h_kv + kPagedThreads / 32 - 1) / (kPagedThreads / 32), 8ll * h->shared.sms);
        const auto kernel = h->d.d_h == 64 ? paged_read_blocks_kernel<64> : h->d.d_h == 128 ? paged_read_blocks_kernel<128> : paged_read_blocks_kernel<256>;
        return launched(launch(kernel, p, dim3(grid), dim3(kPagedThreads), (B + 1) * 4, st, 1, h->pdl));
    }
    if (T <= 16 * h->shared.sms) return launched(launch(paged_read_kernel<1>, p, dim3(T), dim3(kPagedThreads), 0, st, 1, h->pdl));
    return launched(launch(paged_read_kernel<8>, p, dim3((T + 7) / 8), dim3(kPagedThreads), 0, st, 1, h->pdl));
}

namespace {

struct AttnPlan { bool tiles; int32_t group, rows, row_blocks, grid; size_t split_at, bytes; };   // rows: of a segment
// The launch of an attention call, from what the host knows of it; false for bad arguments.
bool attn_plan(qlinear_paged_t h, int32_t h_q, int32_t B, int32_t max_q, AttnPlan* a)
{
    if (!h || h_q < 1 || h_q > 65536 || h_q % h->d.h_kv || B < 0 || B > QL_PAGED_MAX_SEQUENCES || max_q < 0) return false;
    a->group = h_q / h->d.h_kv;
    const int64_t rows = (int64_t)max_q * a->group;
    if (rows > INT32_MAX / 2) return false;
    a->tiles = rows > attn_max_rows(h->d.d_h);
    a->rows = a->tiles ? (h->d.d_h == 256 ? TileShape<256>::kRows : TileShape<128>::kRows) : kAttnCols;
    a->row_blocks = (int32_t)((rows + a->rows - 1) / a->rows);
    a->grid = (a->tiles || B > h->two_ctas_upto ? 1 : 2) * h->shared.sms;   // (every CTA at once: spans of equal length in two rounds take a round's start and end more)
    const size_t most = (size_t)(a->tiles ? 1 : 2) * h->shared.sms;      // (whatever B: a workspace for many sequences serves fewer)
    a->split_at = 2 * most * a->rows * (h->d.d_h + 2) * sizeof(float);
    a->bytes = a->split_at + most * sizeof(int4);
    return true;
}

template <int D, AttnCap CAP>
cudaError_t launch_attention_as(const PagedAttnParams& p, bool tiles, int device, cudaStream_t st, bool pdl)
{
    using T = TileShape<D>;
    static std::atomic<bool> flags[64];
    constexpr int kMost = attn_smem<D>(QL_PAGED_MAX_SEQUENCES), kMostTiles = 1024 + T::kOffPre + (QL_PAGED_MAX_SEQUENCES + 1) * 4;
    if (!flags[device].load(std::memory_order_acquire)) {
        cudaError_t e = cudaFuncSetAttribute(paged_attention_kernel<D, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_tiles_kernel<D, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostTiles);
        cudaFuncAttributes at;
        if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, paged_tiles_kernel<D, CAP>);
        if (e != cudaSuccess) return e;
        if (at.numRegs < kTileRegisters) return cudaErrorInvalidConfiguration;   // (the roles' shares come from what the block was launched with: they would be waited for)
        flags[device].store(true, std::memory_order_release);
    }
    cudaError_t e = tiles ? launch(paged_tiles_kernel<D, CAP>, p, dim3(p.grid), dim3(kTileThreads), 1024 + T::kOffPre + (p.batch.B + 1) * 4, st, 1, pdl)
                          : launch(paged_attention_kernel<D, CAP>, p, dim3(p.grid), dim3(kAttnWarps * 32), attn_smem<D>(p.batch.B), st, 1, pdl);
    if (e != cudaSuccess) return e;
    return tiles ? launch(paged_combine_kernel<D, T::kRows, 4, 1>, p, dim3(p.grid, T::kRows / 32), dim3(256), 0, st, 1, pdl)
                 : launch(paged_combine_kernel<D, kAttnCols, 1, 4>, p, dim3(p.grid, (std::min(kAttnCols, p.max_q * p.group) + 1) / 2), dim3(256), 0, st, 1, pdl);
}

template <int D>
cudaError_t launch_attention(const PagedAttnParams& p, bool tiles, int device, cudaStream_t st, bool pdl)
{
    if (!(p.softcap > 0.f)) return launch_attention_as<D, kCapNone>(p, tiles, device, st, pdl);
    return p.softcap <= kMostPlainCap ? launch_attention_as<D, kCapPlain>(p, tiles, device, st, pdl) : launch_attention_as<D, kCapHigh>(p, tiles, device, st, pdl);
}

}  // namespace

extern "C" size_t qlinear_paged_attention_workspace(qlinear_paged_t h, int32_t h_q, int32_t B, int32_t max_q)
{
    AttnPlan a;
    return attn_plan(h, h_q, B, max_q, &a) ? a.bytes : 0;
}

namespace {
template <int D> int ctas_that_fit(int32_t B)
{
    int least = INT_MAX;
    for (const auto kernel : {paged_attention_kernel<D, kCapNone>, paged_attention_kernel<D, kCapPlain>, paged_attention_kernel<D, kCapHigh>}) {
        int fit = -1;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, attn_smem<D>(QL_PAGED_MAX_SEQUENCES)) != cudaSuccess ||
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, kernel, kAttnWarps * 32, attn_smem<D>(B)) != cudaSuccess) { cudaGetLastError(); return -1; }
        least = std::min(least, fit);
    }
    return least;
}
}  // namespace

extern "C" int32_t qlinear_debug_paged_ctas(qlinear_paged_t h, int32_t B, int32_t* fit)
{
    AttnPlan a;
    if (!h || !fit || !attn_plan(h, h->d.h_kv, B, 1, &a)) return 0;
    DeviceGuard guard(h->device);
    *fit = !guard.ok ? -1 : h->d.d_h == 64 ? ctas_that_fit<64>(B) : h->d.d_h == 128 ? ctas_that_fit<128>(B) : ctas_that_fit<256>(B);
    return a.grid / h->shared.sms;
}

extern "C" ql_status qlinear_paged_attention(qlinear_paged_t h, const void* q, int64_t q_ld, void* out, int64_t out_ld, int32_t h_q, const int32_t* table, int64_t table_ld, int32_t table_width,
                                             const int32_t* kv_len, const int32_t* q_start, int32_t B, int32_t T, int32_t max_q, float scale, float softcap, int32_t window,
                                             void* workspace, size_t workspace_bytes, void* stream)
{
    PagedAttnParams p{};
    AttnPlan a;
    if (!batch_of(h, table, table_ld, table_width, kv_len, q_start, B, T, &p.batch) || !attn_plan(h, h_q, B, max_q, &a)) return QL_ERR_INVALID_ARG;
    if (!(std::fabs(scale) <= kMostScale) || !(softcap >= 0.f) || !std::isfinite(softcap) || window < 0) return QL_ERR_INVALID_ARG;
    if (B == 0 || T == 0 || max_q == 0) return QL_OK;
    {   // the kernels number the steps of a KV head's segments in 32 bits
        const int64_t held = std::min((int64_t)table_width * h->d.page_size, (int64_t)INT32_MAX);
        const int64_t segments = a.tiles ? std::min((int64_t)B * a.row_blocks, (int64_t)T * a.group / a.rows + B) : B;
        if (segments * (a.tiles ? held / TileShape<128>::N + 1 + kTileOverhead : held / kPagedBlock + 1 + kAttnOverhead) > INT32_MAX) return QL_ERR_INVALID_ARG;
    }
    const int32_t d = h->d.d_h;
    if (!rows_ok(q, q_ld, (int64_t)h_q * d) || !rows_ok(out, out_ld, (int64_t)h_q * d) || q == out) return QL_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 32) || workspace_bytes < a.bytes) return QL_ERR_INVALID_ARG;
    if (timed_out(h)) return QL_ERR_DEVICE_TIMEOUT;
    DeviceGuard guard(h->device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    p.q = static_cast<const __half*>(q);
    p.out = static_cast<__half*>(out);
    p.partial = static_cast<float*>(workspace);
    p.split = reinterpret_cast<int4*>(static_cast<char*>(workspace) + a.split_at);
    p.q_ld = q_ld; p.out_ld = out_ld;
    p.h_q = h_q; p.group = a.group; p.max_q = max_q; p.row_blocks = a.row_blocks; p.window = window;
    p.scale = scale; p.grid = a.grid;
    // (a cap below makes all scores one to 30 digits, a cap above leaves them what they are)
    p.softcap = softcap > 0.f ? std::min(std::max(softcap, 1e-30f * std::max(std::fabs(scale), 1.f)), 1e38f) : 0.f;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto go = d == 64 ? launch_attention<64> : d == 128 ? launch_attention<128> : launch_attention<256>;
    return launched(go(p, a.tiles, h->device, st, h->pdl));
}

// ---------------------------------------------------------------------------------------------------- logits
namespace {

template <typename T>
cudaError_t launch_logits(LogitsParams p, int device, int sms, cudaStream_t st)
{
    constexpr int TILE = sizeof(T) == 2 ? 2048 : 1024, kPiece = 4 * kLogitsThreads * 16 / (int)sizeof(T);
    static std::atomic<bool> flags[64];
    if (!flags[device].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(adjust_seen_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSeenBytes);
        if (e != cudaSuccess) return e;
        flags[device].store(true, std::memory_order_release);
    }
    const bool pdl = pdl_enabled(), some = p.tokens || p.bias_ids;
    const unsigned tiles = pieces(p.vocab, TILE);
    // one launch until its CTAs fill the SMs a few times over: each goes through its row's whole history (rows of 128256, history of 1280, one launch / two: 1 row 5.6 / 7.4 us,
    // 8 rows 6.4 / 7.4, 16 rows 7.8 / 8.2, 256 rows 79 / 29)
    if (some && (int64_t)p.rows * tiles <= 4 * sms)
        return launch(adjust_logits_kernel<T, TILE>, p, dim3(tiles, p.rows), dim3(kLogitsThreads), TILE * 8, st, 1, pdl);
    p.masked = p.mask || p.x != p.y;
    cudaError_t e = cudaSuccess;
    if (p.masked) e = launch(mask_logits_kernel<T>, p, dim3(pieces(p.vocab, kPiece), p.rows), dim3(kLogitsThreads), 0, st, 1, pdl);
    if (e == cudaSuccess && some) e = launch(adjust_seen_kernel<T>, p, dim3(pieces(p.vocab, kSeenTokens), p.rows), dim3(kSeenThreads), kSeenBytes, st, 1, pdl);
    return e;
}

}  // namespace

extern "C" ql_status qlinear_adjust_logits(const void* logits, int64_t ld, void* out, int64_t out_ld, int32_t rows, int32_t vocab, int32_t is_fp32,
                                           const int32_t* tokens, int32_t n_tokens, const int32_t* start, const int32_t* n_prompt,
                                           const float* repetition, const float* presence, const float* frequency,
                                           const int32_t* bias_ids, const float* bias_values, const int32_t* bias_start, int32_t n_biases,
                                           const void* mask, int64_t mask_ld, int32_t device, void* stream)
{
    if (rows < 0 || rows > 65535 || vocab < 1 || (is_fp32 != 0 && is_fp32 != 1) || n_tokens < 0 || n_biases < 0 || device < 0) return QL_ERR_INVALID_ARG;
    const uintptr_t size = is_fp32 ? 4 : 2;
    if (rows == 0) return QL_OK;
    if (!logits || !out || !aligned(logits, size) || !aligned(out, size) || ld < vocab || out_ld < vocab || (logits == out && ld != out_ld)) return QL_ERR_INVALID_ARG;
    if ((tokens && !start) || (n_tokens > 0 && !tokens) || (bias_ids && (!bias_values || !bias_start)) || (n_biases > 0 && !bias_ids) || (mask && mask_ld < ((int64_t)vocab + 31) / 32)) return QL_ERR_INVALID_ARG;
    for (const void* p : {(const void*)tokens, (const void*)start, (const void*)n_prompt, (const void*)repetition, (const void*)presence, (const void*)frequency, (const void*)bias_ids,
                          (const void*)bias_values, (const void*)bias_start, mask})
        if (!aligned(p, 4)) return QL_ERR_INVALID_ARG;
    int sms;
    const ql_status ready = device_sms(device, &sms);
    if (ready != QL_OK) return ready;
    DeviceGuard guard(device);
    if (!guard.ok) { cudaGetLastError(); return QL_ERR_CUDA; }
    LogitsParams p{};
    p.x = logits; p.y = out; p.ld = ld; p.out_ld = out_ld; p.mask_ld = mask_ld;
    p.tokens = tokens; p.start = start; p.n_prompt = n_prompt;
    p.repetition = repetition; p.presence = presence; p.frequency = frequency;
    p.bias_ids = bias_ids; p.bias_values = bias_values; p.bias_start = bias_start;
    p.mask = static_cast<const uint32_t*>(mask);
    p.rows = rows; p.vocab = vocab; p.n_tokens = n_tokens; p.n_biases = n_biases;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return launched(is_fp32 ? launch_logits<float>(p, device, sms, st) : launch_logits<__half>(p, device, sms, st));
}
