// Pages chosen for a query: what a page's keys reach per channel, held in 8 bits, and the pages whose bounds promise the largest scores.
//
// Of a page's tokens and a KV head, with hi_c and lo_c the largest and the smallest key element of channel c (fp16(q s), as the cache stands for), top = max_c max(hi_c, -lo_c):
//     scale = top / 127,   r = 127 / top,   bounds = min(127, ceil(hi_c r)), max(-127, floor(lo_c r))                                      (IEEE fp32; top 0: all zero)
// A query q reaches at most sum_c max(q_c hi_c, q_c lo_c) = sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c with any token of the page; summed over the `group` query heads that read a KV head
// this is one product of 2 d numbers, whatever the group.  So for a row and KV head: Q+ and Q- the sums over the heads of max(q, 0) and min(q, 0) (fp32, in the heads' order),
// in whole numbers of 1 / 32767 of the largest magnitude, r' = 32767 / top', rint(Q r'); the score of a page is
//     fp32(sum_c Q+_c hi_c + Q-_c lo_c) * scale                                                         (the sum exact: below 2^31 for 512 products)
// and every number on the way is defined to the bit, so the choice is, ties included.  A score that is no number (keys beyond fp16 leave an infinite scale: 0 * inf) comes behind all others.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <limits.h>
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
__device__ __forceinline__ long long bounds_scan(long long v, long long* total, long long* sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long run = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += u;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = run;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kBoundsWarps; ++w) {
        if (w == warp) before = all;
        all += sums[w];
    }
    *total = all;
    return run - v + before;
}

// A warp takes a page and KV head: in a block of 16 tokens lane 4 t + c has eight elements of each group of the tokens t and t + 8, so that the maxima over tokens are packed fp16
// instructions on what it holds, and at the end (the smallest as the largest of the negated: one operation for both) 8 lanes share the values out among them: each exchange halves what a lane goes on with (28
// exchanges for 32 pairs, not 96), and a lane is left with elements in a row, which it encodes and stores.
// Every CTA numbers the touched columns of the batch (a scan) and takes pages in turn, 32 of them looked up side by side.
// Bound: instruction issue (68 % of the slots: 22 instructions for eight elements, half of them the unpack): the keys of 29500 tokens, 8 heads of 128, in 12.7 us (17 MB read, 2.6 at the copy rate), 14 with two blocks' loads
// in flight or their lines prefetched; for a generated token a sequence (7.3 us) the chain length -> column -> page -> keys.
template <int D>
__global__ void __launch_bounds__(kBoundsThreads, D == 256 ? 2 : 4) paged_bounds_kernel(const PagedBoundsParams p)
{
    constexpr int NB = D / 64, kBlock = paged_block_bytes(D), kPairs = 16 * NB;   // pairs of elements of a lane: largest and smallest
    extern __shared__ int pre[];                                         // [B + 1] touched columns before sequence b, [B] the first of them, [B] its length
    __shared__ long long sums[kBoundsWarps];
    __shared__ int theirs[kBoundsWarps][32];
    __shared__ int3 looked_up[kBoundsWarps][32];                         // page, column, tokens in it: of 32 pages of the CTA (in registers beside the maxima they would spill)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const PagedBatch& bt = p.batch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t = lane >> 2, c = lane & 3, log2_page = bt.log2_blocks + 4;
    int *first_of = pre + bt.B + 1, *len_of = first_of + bt.B;
    long long columns = 0;
    if (tid == 0) pre[0] = 0;
    for (int b0 = 0; b0 < bt.B; b0 += kBoundsThreads) {
        const int b = b0 + tid;
        int first = 0;
        long long all;
        const int n = b < bt.B ? touched_columns(bt, b, &first) : 0;
        const long long before = bounds_scan(n, &all, sums);
        if (b < bt.B) { pre[b + 1] = (int)(columns + before + n); first_of[b] = first; len_of[b] = bt.kv_len[b]; }
        columns += all;
    }
    if (columns > INT_MAX) return;                                       // (rows named more than once, against the rules: they lie in T / page_size + 2 B columns at most)
    const int total = (int)columns;
    __syncthreads();
    const auto tokens_in = [&](int len, int column) { return (int)min((int64_t)len - ((int64_t)column << log2_page), (int64_t)1 << log2_page); };
    const int mine = total > (int)blockIdx.x ? (total - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;   // pages of this CTA: blockIdx.x, + gridDim.x, ...
    for (int base = 0; base < mine; base += 32) {
        __syncwarp();
        if (base + lane < mine) {
            const int k = (int)blockIdx.x + (base + lane) * (int)gridDim.x;
            int b = 0, hi_b = bt.B;                                      // pre[b] <= k < pre[hi_b]
            while (hi_b - b > 1) {
                const int mid = (b + hi_b) >> 1;
                if (pre[mid] <= k) b = mid;
                else hi_b = mid;
            }
            const int column = first_of[b] + k - pre[b];
            looked_up[warp][lane] = make_int3(bt.table[b * bt.table_ld + column], column, tokens_in(len_of[b], column));
        }
        __syncwarp();
        const int tasks = min(32, mine - base) * bt.h_kv;
        for (int task = warp; task < tasks; task += kBoundsWarps) {
            const int at = task / bt.h_kv, head = task - at * bt.h_kv, page = looked_up[warp][at].x, tokens = looked_up[warp][at].z;
            if (page < 0 || page >= bt.n_pages) continue;
            const uint8_t* blk = bt.pool + (((int64_t)page * bt.h_kv + head) << bt.log2_blocks) * kBlock;
            // Of the sequences that end in a page the one with the most tokens there speaks for it (those with as many say the same).  A lane's last entry of one with more in this column is on its way until the keys are done, to
            // shared memory: waited for before them a generated token a sequence takes 1.8 us more, in a register prompts do, which spill then.
            const bool partly = tokens < 1 << log2_page;
            if (partly) {
                const int column = looked_up[warp][at].y;
                bool requested = false;
                for (int b = lane; b < bt.B; b += 32) {
                    if (column < first_of[b] || column - first_of[b] >= pre[b + 1] - pre[b] || tokens_in(len_of[b], column) <= tokens) continue;
                    if (requested) {
                        asm volatile("cp.async.wait_all;" ::: "memory");
                        if (theirs[warp][lane] == page) break;
                    }
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(&theirs[warp][lane])), "l"(bt.table + b * bt.table_ld + column) : "memory");
                    requested = true;
                }
                if (!requested) theirs[warp][lane] = -1;
            }
            uint32_t top[kPairs];                                        // pairs 4 (4 j + 2 e + s) ..: panel j, group e, s: of the negated
#pragma unroll
            for (int i = 0; i < kPairs; ++i) top[i] = i & 4 ? 0x7c007c00u : 0xfc00fc00u;   // (infinities)
            const auto take = [&](uint32_t word, uint32_t scale, uint32_t* to) {
                uint32_t h[4];
                unpack_int4_word(word, h);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t v = h2_mul(h[i], scale);
                    const __half2 a = __hmax2(*reinterpret_cast<const __half2*>(to + i), *reinterpret_cast<const __half2*>(&v)), b = __hmin2(*reinterpret_cast<const __half2*>(to + 4 + i), *reinterpret_cast<const __half2*>(&v));
                    to[i] = *reinterpret_cast<const uint32_t*>(&a);
                    to[4 + i] = *reinterpret_cast<const uint32_t*>(&b);
                }
            };
#pragma unroll 1
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
                        take(kw[j].x, __byte_perm(ks[j].x, ks[j].x, 0x1010), top + 16 * j);
                        take(kw[j].y, __byte_perm(ks[j].y, ks[j].y, 0x1010), top + 16 * j + 8);
                    }
                    if (t0 + t + 8 < tokens) {
                        take(kw[j].z, __byte_perm(ks[j].x, ks[j].x, 0x3232), top + 16 * j);
                        take(kw[j].w, __byte_perm(ks[j].y, ks[j].y, 0x3232), top + 16 * j + 8);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kPairs; ++i) top[i] ^= i & 4 ? 0x80008000u : 0u;   // (of the negated, the largest)
            // the lane with t keeps the pairs kPairs / 8 * t ..
            int held = kPairs;
#pragma unroll
            for (int o = 16; o >= 4; o >>= 1) {
                held >>= 1;
#pragma unroll
                for (int i = 0; i < kPairs / 2; ++i) {
                    if (i >= held) break;
                    const bool high = lane & o;
                    const uint32_t send = high ? top[i] : top[i + held], keep = high ? top[i + held] : top[i], got = __shfl_xor_sync(0xffffffffu, send, o);
                    const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&keep), *reinterpret_cast<const __half2*>(&got));
                    top[i] = *reinterpret_cast<const uint32_t*>(&m);
                }
            }
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < kPairs / 8; ++i) most = fmaxf(most, fmaxf(__low2float(*reinterpret_cast<const __half2*>(top + i)), __high2float(*reinterpret_cast<const __half2*>(top + i))));
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            if (partly) {
                asm volatile("cp.async.wait_all;" ::: "memory");
                if (__any_sync(0xffffffffu, theirs[warp][lane] == page)) continue;
            }
            const float r = most > 0.f ? __fdiv_rn(127.f, most) : 0.f;
            int8_t* to = p.bounds + ((int64_t)page * bt.h_kv + head) * (2 * D);
#pragma unroll
            for (int i0 = 0; i0 < kPairs / 8; i0 += 2) {                 // four elements to a store
                const int pair = kPairs / 8 * t + i0, j = pair >> 4, e = pair >> 3 & 1, s = pair >> 2 & 1;
                uint32_t w = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __half2 two = *reinterpret_cast<const __half2*>(top + i0 + (i >> 1));
                    const int code = min(__float2int_ru(__fmul_rn(i & 1 ? __high2float(two) : __low2float(two), r)), 127);   // (the negated is rounded up: its negative down)
                    w |= ((uint32_t)(s ? -code : code) & 255u) << (8 * i);
                }
                *reinterpret_cast<uint32_t*>(to + s * D + 64 * j + 32 * e + 8 * c + 2 * (pair & 3)) = w;
            }
            if (lane == 0) p.scales[(int64_t)page * bt.h_kv + head] = __fdiv_rn(most, 127.f);
        }
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
    bool gathered;               // the first CTA of a cluster has room for every column's key
};
constexpr int kSelectMostColumns = 1 << 18;
// Keys of columns: 0, no candidate; kNoNumber, a candidate whose score is no number; from 0x007fffff (-inf) to 0xff800000 (inf), scores; kAlways, taken whatever the scores.  No scale, whatever it holds, makes a key
// of another kind, so the kAlways are the first and the recent columns alone, budget of them at most.
constexpr uint32_t kNoNumber = 1, kAlways = 0xffffffffu;
__device__ __forceinline__ uint32_t select_key(int sum, float scale)
{
    const float score = __fadd_rn(__fmul_rn(__int2float_rn(sum), scale), 0.f);   // (-0 becomes 0: equal scores have equal keys)
    const uint32_t bits = __float_as_uint(score);
    return score != score ? kNoNumber : bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

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

constexpr int kSelectThreads = 256, kSelectWarps = kSelectThreads / 32;
constexpr int kSelectGathered = 40 << 10;                                // columns whose keys one CTA holds

__device__ __forceinline__ void cluster_store(uint32_t* p, uint32_t rank, uint32_t v)
{
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}
// Exclusive sum over the CTA's kSelectThreads threads, the whole sum in *total.
__device__ __forceinline__ int select_scan(int v, int* total, int* sums)
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
    const int mine = lane < kSelectWarps ? sums[lane] : 0;
    *total = (int)__reduce_add_sync(0xffffffffu, (unsigned)mine);
    return run - v + (int)__reduce_add_sync(0xffffffffu, lane < warp ? (unsigned)mine : 0u);
}

// The pages of a row and KV head by a cluster.  Each CTA scores a contiguous share of the columns, a warp 32 of them at a time: D / 8 lanes read a page's 2 D bytes, the loads of 8 turns in flight before any is used, and
// the eight sums of a lane are added over those lanes by halves (each lane keeps the half of the sums that is its own: 8 exchanges for 8 sums, not 8 times log2 of the lanes).  Scores become ordered 32-bit keys in
// the shared memory of the cluster's first CTA, which finds the budget-th largest digit by digit (8 bits, from the highest bit in which keys differ; rarely more than two rounds) and writes the columns down in order.  Tables
// too wide for one CTA's shared memory (40960 columns) leave the keys where they are: the CTAs add their histograms through distributed shared memory.
// Bound: the chain length -> page -> bounds -> meeting -> digits, 8 us (10.3 for a row of 8 heads and 2048 pages).  For many rows latency still, with 35 % of the warps active: 64 rows over 512 pages take 22.5 us for 68 MB of bounds, 0.46 of the copy rate (with two CTAs of 512
// threads an SM 27.8); 32 ragged rows use 33 % of the issue slots and 12 % of DRAM.
template <int D>
__global__ void __launch_bounds__(kSelectThreads, 4) paged_select_kernel(const PagedSelectParams p)
{
    constexpr int kLanes = D / 8, kPer = 32 / kLanes, kTurns = 8;        // lanes of a page's 2 D bytes, 16 each; pages at once; loads in flight
    extern __shared__ uint32_t keys[];                                   // [share], or every column's
    __shared__ __align__(16) int16_t codes[2 * D];
    __shared__ int hist[2][256], counts[4], sums[kSelectWarps], found_digit, found_left, found_count;
    __shared__ unsigned long long found;                                 // the row's sequence and position, one more of each
    __shared__ uint32_t range[2];                                        // the complement of the smallest key, the largest
    __shared__ float most[kSelectWarps];
    const PagedBatch& bt = p.batch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, log2_page = bt.log2_blocks + 4;
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const int t = (int)(blockIdx.x / size), head = blockIdx.y;
    if (tid == 0) { found = 0; range[0] = range[1] = 0; }
    if (tid < 4) counts[tid] = 0;
    if (tid < 256) hist[0][tid] = hist[1][tid] = 0;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (a CTA's shared memory is written by others once it has started)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();
    // ---- the sums over the heads, in whole numbers; the row's sequence
    float above = 0.f, below = 0.f;
    if (tid < D) {
        const __half* q = p.q + t * p.q_ld + (int64_t)head * p.group * D + tid;
#pragma unroll 4
        for (int h = 0; h < p.group; ++h) {
            const float x = __half2float(q[(int64_t)h * D]);
            above = __fadd_rn(above, fmaxf(x, 0.f));
            below = __fadd_rn(below, fminf(x, 0.f));
        }
    }
    for (int b = tid; b < bt.B; b += kSelectThreads) {
        int first;
        const int rows = paged_rows(bt, b, &first);
        const int len = bt.kv_len[b];
        if (t >= first && t < first + rows)                              // (the largest: the same for every CTA of the cluster, whatever q_start holds: they meet)
            atomicMax(&found, (unsigned long long)(b + 1) << 32 | (uint32_t)max((int64_t)len - rows + (t - first) + 1, (int64_t)0));
    }
    float m = fmaxf(above, -below);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) most[warp] = m;
    __syncthreads();
    const int seq = (int)(found >> 32) - 1, pos = (int)(uint32_t)found - 1;
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (seq < 0) return;                                                 // (a row of no sequence: the whole cluster leaves)
    m = 0.f;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) m = fmaxf(m, most[w]);
    const float r = m > 0.f ? __fdiv_rn(32767.f, m) : 0.f;
    if (tid < D) {
        codes[tid] = (int16_t)max(min(__float2int_rn(__fmul_rn(above, r)), 32767), -32767);
        codes[D + tid] = (int16_t)max(min(__float2int_rn(__fmul_rn(below, r)), 32767), -32767);
    }
    __syncthreads();

    // ---- the keys of this CTA's columns: 0 for those that are no candidates, the largest number for those that are always taken
    const int last = pos < 0 ? -1 : min(pos >> log2_page, bt.table_width - 1), columns = last + 1;
    const int share = (columns + (int)size - 1) / (int)size, begin = min((int)rank * share, columns), n_mine = min(columns - begin, share);   // (share <= p.share: table_width / size rounded up)
    const bool all = columns <= p.budget;                                // (no scores needed)
    const int sub = lane % kLanes, turn = (sub & kLanes / 2 ? 4 : 0) + (sub & kLanes / 4 ? 2 : 0) + (sub & kLanes / 8 ? 1 : 0);
    const int4 q0 = reinterpret_cast<const int4*>(codes)[2 * sub], q1 = reinterpret_cast<const int4*>(codes)[2 * sub + 1];
    const int8_t* from = p.bounds + 16 * sub;
    const auto put = [&](int at, uint32_t key) {
        if (p.gathered && size > 1) cluster_store(keys + begin + at, 0, key);
        else keys[at] = key;
    };
    const int32_t* row = bt.table + seq * bt.table_ld + begin;
    int page_next = warp * 32 + lane < n_mine ? row[warp * 32 + lane] : -1;
    for (int w0 = warp * 32; w0 < n_mine; w0 += kSelectThreads) {
        const int at = w0 + lane, column = begin + at, page = page_next;
        page_next = at + kSelectThreads < n_mine ? row[at + kSelectThreads] : -1;
        const bool ok = page >= 0 && page < bt.n_pages, always = all || column < p.first || column > last - p.recent;
        if (at < n_mine && (!ok || always)) put(at, ok ? kAlways : 0u);
        if (all) continue;
        const int64_t mine = (int64_t)(ok ? page : 0) * bt.h_kv + head;
        const uint32_t scored = __ballot_sync(0xffffffffu, ok && !always);
        const float scale = scored >> lane & 1 ? p.scales[mine] : 0.f;
#pragma unroll 1
        for (int i0 = 0; i0 < 32; i0 += kTurns * kPer) {
            uint4 u[kTurns];
#pragma unroll
            for (int k = 0; k < kTurns; ++k) {
                const int64_t record = __shfl_sync(0xffffffffu, mine, i0 + k * kPer + lane / kLanes);
                u[k] = *reinterpret_cast<const uint4*>(from + record * (2 * D));
            }
            if (i0 + kTurns * kPer < 32) {                               // (the next turns' are on their way to L2 meanwhile: a lane 128 bytes of a record)
                const int k = lane * kTurns * kPer / 32, line = lane - k * 32 / (kTurns * kPer);
                const int64_t record = __shfl_sync(0xffffffffu, mine, i0 + kTurns * kPer + k);
                if (128 * line < 2 * D) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.bounds + record * (2 * D) + 128 * line));
            }
            int s[kTurns];
#pragma unroll
            for (int k = 0; k < kTurns; ++k) {
                s[k] = __dp2a_lo(q0.x, (int)u[k].x, 0);
                s[k] = __dp2a_hi(q0.y, (int)u[k].x, s[k]);
                s[k] = __dp2a_lo(q0.z, (int)u[k].y, s[k]); s[k] = __dp2a_hi(q0.w, (int)u[k].y, s[k]);
                s[k] = __dp2a_lo(q1.x, (int)u[k].z, s[k]); s[k] = __dp2a_hi(q1.y, (int)u[k].z, s[k]);
                s[k] = __dp2a_lo(q1.z, (int)u[k].w, s[k]); s[k] = __dp2a_hi(q1.w, (int)u[k].w, s[k]);
            }
            int held = kTurns;
#pragma unroll
            for (int o = kLanes / 2; o >= kLanes / 8; o >>= 1) {         // this lane's half of the sums stays
                held >>= 1;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k >= held) break;
                    const bool high = sub & o;
                    const int send = high ? s[k] : s[k + held], keep = high ? s[k + held] : s[k];
                    s[k] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
            }
#pragma unroll
            for (int o = kLanes / 16; o >= 1; o >>= 1) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
            const int src = i0 + turn * kPer + lane / kLanes;            // the column (of the 32) whose sum this lane has
            const float unit = __shfl_sync(0xffffffffu, scale, src);
            if ((scored >> src & 1) && sub % (kLanes / 8) == 0) put(w0 + src, select_key(s[0], unit));
        }
    }

    // ---- who looks for the threshold: the first CTA, which has every key, or, where they do not fit, the cluster
    const bool together = !p.gathered && size > 1;
    int n = n_mine, lo = begin;
    if (p.gathered && size > 1) {
        cluster_meet();
        if (rank > 0) return;
        n = columns;
        lo = 0;
    }
    const uint32_t parts = together ? size : 1;
    const auto meet = [&]() {
        if (together) cluster_meet();
        else __syncthreads();
    };
    const auto sum_of = [&](const int* v) {                              // over the parts
        if (!together) return *v;
        int x[8], sum = 0;
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) x[k] = k < parts ? cluster_load(v, k) : 0;
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) sum += x[k];
        return sum;
    };
    __syncthreads();
    uint32_t least = 0, largest = 0;                                     // (of the complements; of the keys)
    int candidates = 0, always = 0;
    for (int i = tid; i < n; i += kSelectThreads) {
        const uint32_t key = keys[i];
        candidates += key != 0;
        always += key == kAlways;
        if (key == 0 || key == kAlways) continue;
        least = max(least, ~key);
        largest = max(largest, key);
    }
    candidates = __reduce_add_sync(0xffffffffu, candidates);
    always = __reduce_add_sync(0xffffffffu, always);
    least = __reduce_max_sync(0xffffffffu, least);
    largest = __reduce_max_sync(0xffffffffu, largest);
    if (lane == 0) {
        atomicAdd(&counts[0], candidates);
        atomicAdd(&counts[1], always);
        atomicMax(&range[0], least);
        atomicMax(&range[1], largest);
    }
    meet();
    candidates = sum_of(&counts[0]);
    always = sum_of(&counts[1]);
    least = range[0];
    largest = range[1];
    if (together)
        for (uint32_t k = 0; k < parts; ++k) {
            least = max(least, (uint32_t)cluster_load(reinterpret_cast<const int*>(&range[0]), k));
            largest = max(largest, (uint32_t)cluster_load(reinterpret_cast<const int*>(&range[1]), k));
        }

    // ---- the threshold: every key above it is taken, and `left` of those that equal it
    uint32_t threshold = 0;
    int left = 0;
    if (candidates > p.budget) {
        const uint32_t base = ~least;
        left = p.budget - always;                                        // (not below 0: first + recent <= budget)
        uint32_t prefix = 0;                                             // of key - base
        int shift = 32 - __clz(largest - base), bits = 0;
        threshold = left > 0 ? base : kAlways - 1;                       // (left 0: those that are always taken are the budget; all keys equal: no rounds)
        for (int round = 0; left > 0 && shift > 0; ++round) {
            bits = min(shift, 8);
            shift -= bits;
            int* h = hist[round & 1];
            for (int i = tid; i < n; i += kSelectThreads) {
                const uint32_t key = keys[i];
                if (key == 0 || key == kAlways) continue;
                const uint32_t x = (key - base) >> shift;
                if (round == 0 || x >> bits == prefix) atomicAdd(&h[x & ((1u << bits) - 1)], 1);
            }
            meet();
            const int sum = tid < 256 ? sum_of(&h[255 - tid]) : 0;       // (thread 0: the largest digit)
            int every;
            const int before = select_scan(sum, &every, sums);
            if (before < left && before + sum >= left) { found_digit = 255 - tid; found_left = left - before; found_count = sum; }
            if (tid < 256) hist[(round + 1) & 1][tid] = 0;               // (its readers are past the meeting above)
            __syncthreads();
            prefix = prefix << bits | (uint32_t)found_digit;
            left = found_left;
            threshold = base + (prefix << shift);
            if (left == found_count) {                                   // all of this digit: no need to tell them apart
                threshold -= 1;
                left = 0;
                break;
            }
        }
    }

    // ---- the columns, in order: where this CTA's begin
    int over = 0, equal = 0;
    const int per = (n + kSelectThreads - 1) / kSelectThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    for (int i = i0; i < i1; ++i) {
        over += keys[i] > threshold;
        equal += left > 0 && keys[i] == threshold;
    }
    int all_over, all_equal;
    int over_at = select_scan(over, &all_over, sums), equal_at = select_scan(equal, &all_equal, sums);
    int over_all = all_over, equal_all = all_equal;
    if (together) {
        if (tid == 0) { counts[2] = all_over; counts[3] = all_equal; }
        cluster_meet();
        over_all = equal_all = 0;
        for (uint32_t k = 0; k < parts; ++k) {
            const int a = cluster_load(&counts[2], k), b = cluster_load(&counts[3], k);
            if (k < rank) { over_at += a; equal_at += b; }
            over_all += a;
            equal_all += b;
        }
    }
    int32_t* to = p.pages + ((int64_t)t * bt.h_kv + head) * p.budget;
    for (int i = i0; i < i1; ++i) {
        const uint32_t key = keys[i];
        const bool is_over = key > threshold, is_equal = left > 0 && key == threshold;
        if (is_over || (is_equal && equal_at < left)) to[over_at + min(equal_at, left)] = lo + i;
        over_at += is_over;
        equal_at += is_equal;
    }
    const int mine = together ? (int)rank : 0;
    for (int i = over_all + min(equal_all, left) + mine * kSelectThreads + tid; i < p.budget; i += (int)parts * kSelectThreads) to[i] = -1;
    if (together) cluster_meet();                                        // (nobody leaves while another reads its counts)
}

}  // namespace ql
