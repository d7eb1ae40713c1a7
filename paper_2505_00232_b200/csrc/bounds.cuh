// Pages chosen for a query: what a page's keys reach per channel, held in 8 bits, and the pages whose bounds promise the largest scores.
//
// Of a page's tokens and a KV head, with hi_c and lo_c the largest and the smallest key element of channel c (fp16(q s), as the cache stands for), top = max_c max(hi_c, -lo_c):
//     scale = top / 127,   r = 127 / top,   bounds = min(127, ceil(hi_c r)), max(-127, floor(lo_c r))                                      (IEEE fp32; top 0: all zero)
// A query q reaches at most sum_c max(q_c hi_c, q_c lo_c) = sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c with any token of the page; summed over the `group` query heads that read a KV head
// this is one product of 2 d numbers, whatever the group.  So for a row and KV head: Q+ and Q- the sums over the heads of max(q, 0) and min(q, 0) (fp32, in the heads' order),
// in whole numbers of 1 / 32767 of the largest magnitude, r' = 32767 / top', rint(Q r'); the score of a page is
//     fp32(sum_c Q+_c hi_c + Q-_c lo_c) * scale                                                         (the sum exact: below 2^31 for 512 products)
// and every number on the way is defined to the bit, so the choice is, ties included.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dequant.cuh"
#include "paged.cuh"

namespace ql {

constexpr int kBoundsThreads = 256, kBoundsWarps = kBoundsThreads / 32;

struct PagedBoundsParams {
    PagedBatch batch;
    int8_t* bounds;              // [n_pages, h_kv, 2, d]: the largest, the smallest
    float* scales;               // [n_pages, h_kv]
};

// The columns of sequence b that its rows lie in: *first the first of them.
__device__ __forceinline__ int touched_columns(const PagedBatch& p, int b, int* first)
{
    int t0;
    const int rows = paged_rows(p, b, &t0), len = p.kv_len[b], log2_page = p.log2_blocks + 4;
    *first = 0;
    if (rows <= 0 || len <= 0) return 0;
    *first = (int)(max((int64_t)len - rows, (int64_t)0) >> log2_page);
    return max(min(((len - 1) >> log2_page) + 1, p.table_width) - *first, 0);
}
// Exclusive sum over the CTA's kBoundsThreads threads, the whole sum in *total.
__device__ __forceinline__ int bounds_scan(int v, int* total, int* sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int run = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += u;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = run;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kBoundsWarps; ++w) {
        if (w == warp) before = all;
        all += sums[w];
    }
    *total = all;
    return run - v + before;
}

// A warp takes a page and KV head: in a block of 16 tokens lane 4 t + c has eight elements of each group of the tokens t and t + 8, so that the maxima over tokens are packed fp16
// instructions on what it holds and three exchanges at the end.  Every CTA numbers the touched columns of the batch (a scan) and takes pages in turn.
// Bound: HBM (the keys of the touched pages, once).
template <int D>
__global__ void __launch_bounds__(kBoundsThreads) paged_bounds_kernel(const PagedBoundsParams p)
{
    constexpr int NB = D / 64, kBlock = paged_block_bytes(D);
    extern __shared__ int pre[];                                         // [B + 1] touched columns before sequence b
    __shared__ int sums[kBoundsWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const PagedBatch& bt = p.batch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t = lane >> 2, c = lane & 3, log2_page = bt.log2_blocks + 4;
    int total = 0;
    if (tid == 0) pre[0] = 0;
    for (int b0 = 0; b0 < bt.B; b0 += kBoundsThreads) {
        const int b = b0 + tid;
        int first, all;
        const int n = b < bt.B ? touched_columns(bt, b, &first) : 0, before = bounds_scan(n, &all, sums);
        if (b < bt.B) pre[b + 1] = total + before + n;
        total += all;
    }
    __syncthreads();
    for (int64_t item = (int64_t)blockIdx.x * kBoundsWarps + warp; item < (int64_t)total * bt.h_kv; item += (int64_t)gridDim.x * kBoundsWarps) {
        const int k = (int)(item / bt.h_kv), head = (int)(item - (int64_t)k * bt.h_kv);
        int b = 0, hi_b = bt.B;                                          // pre[b] <= k < pre[hi_b]
        while (hi_b - b > 1) {
            const int mid = (b + hi_b) >> 1;
            if (pre[mid] <= k) b = mid;
            else hi_b = mid;
        }
        int first;
        touched_columns(bt, b, &first);
        const int column = first + k - pre[b], page = bt.table[b * bt.table_ld + column];
        if (page < 0 || page >= bt.n_pages) continue;
        const int tokens = (int)min((int64_t)bt.kv_len[b] - ((int64_t)column << log2_page), (int64_t)1 << log2_page);
        const uint8_t* blk = bt.pool + (((int64_t)page * bt.h_kv + head) << bt.log2_blocks) * kBlock;
        const uint32_t kMinusInf = 0xfc00fc00u, kPlusInf = 0x7c007c00u;
        uint32_t top[NB][2][4], low[NB][2][4];                           // two elements each
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) { top[j][e][i] = kMinusInf; low[j][e][i] = kPlusInf; }
        const auto take = [&](uint32_t word, uint32_t scale, uint32_t* hi, uint32_t* lo) {
            uint32_t h[4];
            unpack_int4_word(word, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t v = h2_mul(h[i], scale);
                const __half2 x = *reinterpret_cast<const __half2*>(&v);
                const __half2 m = __hmax2(*reinterpret_cast<__half2*>(hi + i), x), n = __hmin2(*reinterpret_cast<__half2*>(lo + i), x);
                hi[i] = *reinterpret_cast<const uint32_t*>(&m);
                lo[i] = *reinterpret_cast<const uint32_t*>(&n);
            }
        };
#pragma unroll 2
        for (int t0 = 0; t0 < tokens; t0 += kPagedBlock, blk += kBlock) {
            uint4 kw[NB];
            uint2 ks[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                kw[j] = *reinterpret_cast<const uint4*>(blk + 512 * j + 16 * lane);
                ks[j] = *reinterpret_cast<const uint2*>(blk + paged_k_scales(D) + t * (8 * NB) + 8 * j);
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if (t0 + t < tokens) {
                    take(kw[j].x, __byte_perm(ks[j].x, ks[j].x, 0x1010), top[j][0], low[j][0]);
                    take(kw[j].y, __byte_perm(ks[j].y, ks[j].y, 0x1010), top[j][1], low[j][1]);
                }
                if (t0 + t + 8 < tokens) {
                    take(kw[j].z, __byte_perm(ks[j].x, ks[j].x, 0x3232), top[j][0], low[j][0]);
                    take(kw[j].w, __byte_perm(ks[j].y, ks[j].y, 0x3232), top[j][1], low[j][1]);
                }
            }
        }
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    __half2 m = *reinterpret_cast<__half2*>(&top[j][e][i]), n = *reinterpret_cast<__half2*>(&low[j][e][i]);
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) {
                        m = __hmax2(m, __shfl_xor_sync(0xffffffffu, m, o));
                        n = __hmin2(n, __shfl_xor_sync(0xffffffffu, n, o));
                    }
                    top[j][e][i] = *reinterpret_cast<const uint32_t*>(&m);
                    low[j][e][i] = *reinterpret_cast<const uint32_t*>(&n);
                    most = fmaxf(most, fmaxf(fmaxf(__low2float(m), __high2float(m)), -fminf(__low2float(n), __high2float(n))));
                }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const float r = most > 0.f ? __fdiv_rn(127.f, most) : 0.f;
        int8_t* to = p.bounds + ((int64_t)page * bt.h_kv + head) * (2 * D);
        // eight elements of a group by one lane each: the lane with t = 4 j + 2 e + (smallest), in turn where there are more of them
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (t == ((4 * j + 2 * e + s) & 7)) {
                        uint32_t w[2] = {0, 0};
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const __half2 two = *reinterpret_cast<const __half2*>(s ? &low[j][e][i >> 1] : &top[j][e][i >> 1]);
                            const float v = __fmul_rn(i & 1 ? __high2float(two) : __low2float(two), r);
                            const int code = s ? max(__float2int_rd(v), -127) : min(__float2int_ru(v), 127);
                            w[i >> 2] |= ((uint32_t)code & 255u) << (8 * (i & 3));
                        }
                        *reinterpret_cast<uint2*>(to + s * D + 64 * j + 32 * e + 8 * c) = make_uint2(w[0], w[1]);
                    }
        if (lane == 0) p.scales[(int64_t)page * bt.h_kv + head] = __fdiv_rn(most, 127.f);
    }
}

struct PagedSelectParams {
    PagedBatch batch;
    const __half* q;
    const int8_t* bounds;
    const float* scales;
    int32_t* pages;              // [T, h_kv, budget]
    int64_t q_ld;
    int32_t group, budget, first, recent, share;                         // share: columns of a CTA at most
};
constexpr int kSelectMostColumns = 1 << 18;

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_meet()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_load(const int* p, uint32_t rank)
{
    uint32_t at;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// The pages of a row and KV head by a cluster, each CTA with a contiguous share of the columns: scores as ordered 32-bit keys in shared memory, the budget-th largest of them digit by digit
// (8 bits, histograms summed through distributed shared memory), then the columns above it, and of those equal to it the first, written down in order.
// Bound: the chain length -> page -> bounds -> four digits, about 6 us; for many rows the bytes of the bounds (2 d + 4 a page and KV head).
template <int D>
__global__ void __launch_bounds__(kBoundsThreads) paged_select_kernel(const PagedSelectParams p)
{
    constexpr int kLanes = D / 8, kPer = 32 / (kLanes < 32 ? kLanes : 32);   // lanes of a page's 2 D bytes, 16 each; pages at once
    static_assert(kLanes <= 32, "");
    extern __shared__ uint32_t keys[];                                   // [share]
    __shared__ __align__(16) int16_t codes[2 * D];
    __shared__ int hist[2][256], counts[4], sums[kBoundsWarps], found_digit, found_left, found_seq;
    __shared__ float most[kBoundsWarps];
    const PagedBatch& bt = p.batch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, log2_page = bt.log2_blocks + 4;
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const int t = (int)(blockIdx.x / size), head = blockIdx.y;
    if (tid == 0) found_seq = -1;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();
    for (int b = tid; b < bt.B; b += kBoundsThreads) {
        int first;
        const int rows = paged_rows(bt, b, &first);
        if (t >= first && t < first + rows) atomicMax(&found_seq, b);    // (the same for every CTA of the cluster, whatever q_start holds: they meet)
    }
    // ---- the sums over the heads, in whole numbers
    float above = 0.f, below = 0.f;
    if (tid < D) {
        const __half* q = p.q + t * p.q_ld + (int64_t)head * p.group * D + tid;
        for (int h = 0; h < p.group; ++h) {
            const float x = __half2float(q[(int64_t)h * D]);
            above = __fadd_rn(above, fmaxf(x, 0.f));
            below = __fadd_rn(below, fminf(x, 0.f));
        }
    }
    float m = fmaxf(above, -below);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) most[warp] = m;
    __syncthreads();
    const int seq = found_seq;
    if (seq < 0) return;                                                 // (a row of no sequence: the whole cluster leaves)
    int t0;
    const int rows_all = paged_rows(bt, seq, &t0), pos = (int)max((int64_t)bt.kv_len[seq] - rows_all + (t - t0), (int64_t)-1);
    m = 0.f;
#pragma unroll
    for (int w = 0; w < kBoundsWarps; ++w) m = fmaxf(m, most[w]);
    const float r = m > 0.f ? __fdiv_rn(32767.f, m) : 0.f;
    if (tid < D) {
        codes[tid] = (int16_t)max(min(__float2int_rn(__fmul_rn(above, r)), 32767), -32767);
        codes[D + tid] = (int16_t)max(min(__float2int_rn(__fmul_rn(below, r)), 32767), -32767);
    }
    hist[0][tid] = hist[1][tid] = 0;
    if (tid < 4) counts[tid] = 0;
    __syncthreads();

    // ---- the keys of this CTA's columns: 0 for those that are no candidates, the largest number for those that are always taken
    const int last = pos < 0 ? -1 : min(pos >> log2_page, bt.table_width - 1), columns = last + 1;
    const int share = (columns + (int)size - 1) / (int)size, lo = min((int)rank * share, columns), n = min(columns - lo, share);   // (share <= p.share: table_width / size rounded up)
    const bool all = columns <= p.budget;                                // (no scores needed)
    int4 q[2];
    q[0] = reinterpret_cast<const int4*>(codes)[2 * (lane % kLanes)];
    q[1] = reinterpret_cast<const int4*>(codes)[2 * (lane % kLanes) + 1];
    const int8_t* from = p.bounds + 16 * (lane % kLanes);
    int candidates = 0;
    for (int w0 = warp * 32; w0 < n; w0 += kBoundsWarps * 32) {
        const int at = w0 + lane, column = lo + at;
        int page = at < n ? bt.table[seq * bt.table_ld + column] : -1;
        const bool ok = page >= 0 && page < bt.n_pages, always = column < p.first || column > last - p.recent;
        uint32_t key = ok ? 0xffffffffu : 0u;
        if (!all) {
            const int64_t mine = ((int64_t)(ok ? page : 0) * bt.h_kv + head);
            const float scale = ok && !always ? p.scales[mine] : 0.f;
            int sum = 0;
#pragma unroll 8
            for (int i = 0; i < 32; i += kPer) {
                const int src = i + lane / kLanes;
                const int64_t record = __shfl_sync(0xffffffffu, mine, src);
                const uint4 u = *reinterpret_cast<const uint4*>(from + record * (2 * D));
                int s = 0;
                s = __dp2a_lo(q[0].x, (int)u.x, s); s = __dp2a_hi(q[0].y, (int)u.x, s);
                s = __dp2a_lo(q[0].z, (int)u.y, s); s = __dp2a_hi(q[0].w, (int)u.y, s);
                s = __dp2a_lo(q[1].x, (int)u.z, s); s = __dp2a_hi(q[1].y, (int)u.z, s);
                s = __dp2a_lo(q[1].z, (int)u.w, s); s = __dp2a_hi(q[1].w, (int)u.w, s);
#pragma unroll
                for (int o = 1; o < kLanes; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                s = __shfl_sync(0xffffffffu, s, (lane % kPer) * kLanes);
                if (lane / kPer == i / kPer) sum = s;
            }
            if (ok && !always) {
                const uint32_t bits = __float_as_uint(__fmul_rn(__int2float_rn(sum), scale) + 0.f);   // (-0 becomes 0: equal scores have equal keys)
                key = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
            }
        }
        if (at < n) keys[at] = key;
        candidates += key != 0;
    }
    candidates = __reduce_add_sync(0xffffffffu, candidates);
    if (lane == 0) atomicAdd(&counts[0], candidates);
    __syncthreads();

    // ---- the threshold: every key above it is taken, and `left` of those that equal it
    uint32_t threshold = 0;
    int left = 0;
    if (!all) {
        uint32_t prefix = 0;
        for (int digit = 0; digit < 4; ++digit) {
            int* h = hist[digit & 1];
            const int shift = 24 - 8 * digit;
            for (int i = tid; i < n; i += kBoundsThreads) {
                const uint32_t key = keys[i];
                if (key != 0 && (digit == 0 || key >> (shift + 8) == prefix)) atomicAdd(&h[key >> shift & 255], 1);
            }
            cluster_meet();
            int sum = 0, total = 0;
            for (uint32_t k = 0; k < size; ++k) sum += cluster_load(&h[255 - tid], k);   // (thread 0: the largest digit)
            if (digit == 0) for (uint32_t k = 0; k < size; ++k) total += cluster_load(&counts[0], k);
            if (digit == 0) left = min(p.budget, total);
            if (digit == 0 && total <= p.budget) { left = 0; break; }    // (every candidate; the whole cluster agrees)
            int every;
            const int before = bounds_scan(sum, &every, sums);
            if (before < left && before + sum >= left) { found_digit = 255 - tid; found_left = left - before; }
            hist[(digit + 1) & 1][tid] = 0;                              // (its readers are past the meeting above)
            __syncthreads();
            prefix = prefix << 8 | (uint32_t)found_digit;
            left = found_left;
        }
        threshold = prefix;
    }

    // ---- the columns, in order: where this CTA's begin
    int over = 0, equal = 0;
    const int per = (n + kBoundsThreads - 1) / kBoundsThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    for (int i = i0; i < i1; ++i) {
        over += keys[i] > threshold;
        equal += threshold != 0 && keys[i] == threshold;
    }
    int all_over, all_equal;
    int over_at = bounds_scan(over, &all_over, sums), equal_at = bounds_scan(equal, &all_equal, sums);
    if (tid == 0) { counts[1] = all_over; counts[2] = all_equal; }
    cluster_meet();
    int over_before = 0, equal_before = 0, over_all = 0, equal_all = 0;
    for (uint32_t k = 0; k < size; ++k) {
        const int a = cluster_load(&counts[1], k), b = cluster_load(&counts[2], k);
        if (k < rank) { over_before += a; equal_before += b; }
        over_all += a;
        equal_all += b;
    }
    over_at += over_before;
    equal_at += equal_before;
    int32_t* to = p.pages + ((int64_t)t * bt.h_kv + head) * p.budget;
    for (int i = i0; i < i1; ++i) {
        const bool is_over = keys[i] > threshold, is_equal = threshold != 0 && keys[i] == threshold;
        if (is_over || (is_equal && equal_at < left)) to[over_at + min(equal_at, left)] = lo + i;
        over_at += is_over;
        equal_at += is_equal;
    }
    for (int i = over_all + min(equal_all, left) + (int)rank * kBoundsThreads + tid; i < p.budget; i += (int)size * kBoundsThreads) to[i] = -1;
    cluster_meet();                                                      // (nobody leaves while another reads its counts)
}

}  // namespace ql
