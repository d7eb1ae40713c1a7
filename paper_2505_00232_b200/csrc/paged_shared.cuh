// Attention over the paged cache for sequences that share their beginning: the beginning of a group's sequences is one stretch of tokens that all rows of the group see whole, what follows it is a
// stretch of each sequence's own.  Both are worked on by the kernels of paged_attention.cuh (few rows) and paged_tiles.cuh (many), whose softmax is one pass with (m, l, o), and joined here:
//   o = sum_parts 2^(m_i - m) o_i / sum_parts 2^(m_i - m) l_i,   m = max m_i
// So 64 sequences of one generated token and 4 query heads a KV head are one tile of 256 rows over the prefix, which is read and unpacked once instead of 64 times.
//
// The plan is a kernel of its own, one CTA: stretches, their lengths as the kernels number their segments, and each row's sequence, from the arrays on the device.  The length of a shared beginning is cut to a
// multiple of 64 tokens (a step of the tiles) and to what all rows of the group see, so that nothing of it needs a mask; what is cut off belongs to what follows, from each sequence's own pages.
//
// 64 sequences of up to 1500 tokens of their own over 32768, 8 KV heads of 128 and 4 queries each: plan 4.8 us, tiles 52 (10 until the first scores are weighed, 28 steps of 1.28, 5 for the sums to leave), few rows 21, join 7;
// qlinear_paged_attention of the same 480.  The sums of cut tiles are 21 MB: laid with eight elements of all rows side by side they leave in 1.7 us less and take the join 1 to 4 more.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "paged.cuh"
#include "paged_attention.cuh"
#include "paged_tiles.cuh"

namespace ql {

constexpr int kSharedThreads = 1024, kMostStretches = QL_PAGED_MAX_SEQUENCES;
constexpr int kStretchUnit = 64;
constexpr int kMostPrefix = 1 << 30;                                     // (positions and rows add up below 2^31)

// A launch of one of the two kernels over the stretches v0 .. v1 - 1.
struct SharedLaunch {
    const float* partial;
    int32_t v0, v1, grid;
    bool tiles;
};
struct SharedPlanParams {
    PagedBatch batch;
    const int32_t* group_start;
    const int32_t* prefix_len;
    int32_t n_groups, group, max_q, tile_rows;
    SharedLaunch prefix, own;    // (the same one, or one each)
    int64_t* spans;              // of a CTA of theirs
    AttnStretch* stretches;      // [n_groups + B]
    int32_t* lengths;            // [n_groups + B + 1]
    int2* row_of;                // [T] the stretches of a served row: its sequence's own, its group's (-1: none); -1: not served
};

template <int kRows>
__device__ __forceinline__ int stretch_length(const AttnStretch& v, int group, bool tiles)
{
    if (!tiles) return v.blocks > 0 ? v.row_blocks * (v.blocks + kAttnOverhead) : 0;
    const int n = (v.rows * group + kRows - 1) / kRows;
    int end, sum = 0;
    if (v.first == 0 && v.pos0 >= v.end - 1) return n * tile_length(stretch_steps<64, kRows>(v, 0, group, &end));   // (every row sees it whole)
    for (int r = 0; r < n; ++r) sum += tile_length(stretch_steps<64, kRows>(v, r * kRows, group, &end));
    return sum;
}

__global__ void __launch_bounds__(kSharedThreads) paged_shared_plan_kernel(const SharedPlanParams p)
{
    __shared__ int start[kMostStretches + 1], len_of[kMostStretches], group_of[kMostStretches], prefix[kMostStretches], sums[32], prefix_length;
    __shared__ unsigned long long every_length;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const PagedBatch& bt = p.batch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = p.n_groups, V = G + bt.B;
    const int64_t held = min((int64_t)bt.table_width << (bt.log2_blocks + 4), (int64_t)INT32_MAX);
    for (int b = tid; b <= bt.B; b += kSharedThreads) start[b] = bt.q_start[b];
    for (int b = tid; b < bt.B; b += kSharedThreads) { len_of[b] = bt.kv_len[b]; group_of[b] = -1; }
    for (int t = tid; t < bt.T; t += kSharedThreads) p.row_of[t] = make_int2(-1, -1);
    int s = 0, e = 0, wanted = 0;                                        // (of this warp's first group, on its way meanwhile)
    if (tid == 0) { prefix_length = 0; every_length = 0; }
    if (warp < G) { s = p.group_start[warp]; e = p.group_start[warp + 1]; wanted = p.prefix_len[warp]; }
    __syncthreads();
    for (int g = warp; g < G; g += kSharedThreads / 32) {
        if (g != warp) { s = p.group_start[g]; e = p.group_start[g + 1]; wanted = p.prefix_len[g]; }
        const bool some = s >= 0 && e <= bt.B && (int64_t)e - s >= 2;
        int64_t least = min(held, (int64_t)kMostPrefix);
        int first = INT32_MAX;                                           // the first sequence with rows
        bool ok = some;
        for (int b = s + lane; some && b < e; b += 32) {
            const int t0 = start[b], t1 = start[b + 1];
            ok = ok && t0 >= 0 && t1 >= t0 && t1 <= bt.T;
            if (t1 <= t0 || len_of[b] <= 0) continue;                    // (a request that is done keeps the others' beginning as it is)
            first = min(first, b);
            least = min(least, (int64_t)len_of[b] - ((int64_t)t1 - t0) + 1);   // what its first row sees
        }
        first = __reduce_min_sync(0xffffffffu, first);
        int sees = __reduce_min_sync(0xffffffffu, (int)max(least, (int64_t)0));
        ok = __all_sync(0xffffffffu, ok) && first != INT32_MAX;
        sees = ok ? max(min(sees, wanted), 0) / kStretchUnit * kStretchUnit : 0;
        for (int b = s + lane; sees > 0 && b < e; b += 32)
            if (len_of[b] > 0) atomicMax(&group_of[b], g);
        if (lane == 0) prefix[g] = sees;
    }
    __syncthreads();
    int before = 0;
    for (int v0 = 0; v0 < V; v0 += kSharedThreads) {
        const int v = v0 + tid;
        int n = 0;
        if (v < V) {
            AttnStretch st{};
            if (v < G) {
                const int sees = prefix[v];
                if (sees > 0) {                                          // (a group of sequences in [0, B))
                    const int s0 = p.group_start[v], e0 = p.group_start[v + 1];
                    int first = s0;
                    while (first + 1 < e0 && (start[first + 1] <= start[first] || len_of[first] <= 0)) ++first;   // the first sequence with rows: its pages
                    st.t0 = start[s0];
                    st.rows = start[e0] - st.t0;
                    st.pos0 = sees - 1;
                    st.end = sees;
                    st.seq = first;
                    st.blocks = sees / kPagedBlock;
                    st.row_blocks = (st.rows * p.group + kAttnCols - 1) / kAttnCols;
                }
            } else {
                const int b = v - G, g = group_of[b], t1 = start[b + 1], len = len_of[b];
                st.t0 = start[b];
                const int rows_all = st.t0 < 0 || t1 > bt.T || t1 < st.t0 ? 0 : t1 - st.t0;
                st.rows = len > 0 ? min(rows_all, p.max_q) : 0;
                st.first = g >= 0 ? prefix[g] : 0;
                st.end = (int)held;
                st.seq = b;
                if (st.rows > 0) {
                    st.pos0 = len - rows_all;
                    const int end = (int)min((int64_t)st.pos0 + st.rows, held);
                    st.blocks = max((int)(((unsigned)max(end, 0) + kPagedBlock - 1) / kPagedBlock) - st.first / kPagedBlock, 0);
                    st.row_blocks = (st.rows * p.group + kAttnCols - 1) / kAttnCols;
                }
                for (int i = 0; i < min(rows_all, p.max_q); ++i) p.row_of[st.t0 + i] = make_int2(v, g);
            }
            p.stretches[v] = st;
            const bool tiles = v < G ? p.prefix.tiles : p.own.tiles;
            n = st.rows <= 0 ? 0 : p.tile_rows == 128 ? stretch_length<128>(st, p.group, tiles) : stretch_length<256>(st, p.group, tiles);
            if (n > 0) atomicAdd(&every_length, (unsigned long long)n);
        }
        int run = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += u;
        }
        __syncthreads();
        if (lane == 31) sums[warp] = run;
        __syncthreads();
        const int mine = sums[lane];
        run += before + (int)__reduce_add_sync(0xffffffffu, lane < warp ? (unsigned)mine : 0u);
        if (v < V) p.lengths[v + 1] = run;
        if (v + 1 == G) prefix_length = run;
        before += (int)__reduce_add_sync(0xffffffffu, (unsigned)mine);
    }
    __syncthreads();
    if (every_length > INT32_MAX) {                                      // rows or sequences named more than once, against the rules: nothing is done
        for (int v = tid; v <= V; v += kSharedThreads) p.lengths[v] = 0;
        for (int t = tid; t < bt.T; t += kSharedThreads) p.row_of[t] = make_int2(-1, -1);
        before = prefix_length = 0;
        __syncthreads();
    }
    if (tid < 2) {
        const SharedLaunch& at = tid == 0 ? p.prefix : p.own;
        const int64_t total = (int64_t)((at.v1 == G ? prefix_length : before) - (at.v0 == G ? prefix_length : 0)) * bt.h_kv;
        p.spans[tid] = max((total + at.grid - 1) / at.grid, (int64_t)(at.tiles ? kSharedTileSpan : kAttnSpan));
    }
    if (tid == 0) p.lengths[0] = 0;
}

struct SharedJoinParams {
    const AttnStretch* stretches;
    const int32_t* lengths;
    const int2* row_of;
    const float* row_o;
    const float2* row_ml;
    __half* out;
    int64_t out_ld;
    int32_t T, h_q, group, h_kv, log2_tile_rows;
    SharedLaunch prefix, own;
    const int64_t* spans;        // of the two launches
};

// The parts of a row in one of its stretches: n of them, in the slots of neighbouring CTAs from c0 on (the first part in slot 1, later ones in slot 0), or, n = 1, in a place of its own.
struct SharedParts { int32_t n, c0, row; };
__device__ __forceinline__ SharedParts shared_parts(const SharedJoinParams& p, bool group_s, int v, int t, int head, int in_group)
{
    const AttnStretch st = p.stretches[v];
    const int32_t v0 = group_s ? p.prefix.v0 : p.own.v0, lengths_v = p.lengths[v], lengths_0 = p.lengths[v0], lengths_1 = p.lengths[group_s ? p.prefix.v1 : p.own.v1];
    const long long span = p.spans[group_s ? 0 : 1];
    const bool tiles = group_s ? p.prefix.tiles : p.own.tiles;
    const int row = (t - st.t0) * p.group + in_group, log2_rows = tiles ? p.log2_tile_rows : 3, block = row >> log2_rows, overhead = tiles ? kTileOverhead : kAttnOverhead;
    int64_t begin = (int64_t)(lengths_v - lengths_0) * p.h_kv;
    int length = 0, end;
    if (st.rows > 0 && tiles && group_s) {                               // (every row sees it whole)
        length = tile_length(st.end / kStretchUnit);
        begin += ((int64_t)block * p.h_kv + head) * length;
    } else if (st.rows > 0 && tiles) {
        const auto steps = [&](int k) { return p.log2_tile_rows == 7 ? stretch_steps<64, 128>(st, k * 128, p.group, &end) : stretch_steps<64, 256>(st, k * 256, p.group, &end); };
        length = tile_length(steps(block));
        for (int k = 0; k < block; ++k) begin += (int64_t)tile_length(steps(k)) * p.h_kv;
        begin += (int64_t)head * length;
    } else if (st.blocks > 0) {
        length = st.blocks + kAttnOverhead;
        begin += ((int64_t)head * st.row_blocks + block) * length;
    }
    SharedParts r{0, 0, row - (block << log2_rows)};
    if (length == 0) return r;
    int c1;                                                              // the CTAs with something of it
    if ((int64_t)(lengths_1 - lengths_0) * p.h_kv <= INT32_MAX) {        // (32 bits: a sixth of the time)
        r.c0 = ((unsigned)begin + overhead) / (unsigned)span;
        c1 = ((unsigned)begin + length - 1) / (unsigned)span;
    } else {
        r.c0 = (int)((begin + overhead) / span);
        c1 = (int)((begin + length - 1) / span);
    }
    r.n = c1 - r.c0 + 1;
    return r;
}

// 8 / W rows (query heads of a KV head) of a token per CTA; W warps share a row's parts, in a fixed order.
template <int D, int W>
__global__ void __launch_bounds__(256) paged_shared_join_kernel(const SharedJoinParams p)
{
    constexpr int V = D / 32;
    __shared__ __align__(16) float sums[8][D];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t = blockIdx.x, head = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % W;
    const int2 of = p.row_of[t];
    if (of.x < 0) return;
    const int r = blockIdx.z * (8 / W) + warp / W;
    float acc[V], l = 0.f, m = -1e30f;
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    if (r < p.group) {
        // (half of the lanes for each of the two)
        SharedParts mine{0, 0, 0};
        if (lane >= 16 || of.y >= 0) mine = shared_parts(p, lane < 16, lane < 16 ? of.y : of.x, t, head, r);
        const SharedParts pre{__shfl_sync(0xffffffffu, mine.n, 0), __shfl_sync(0xffffffffu, mine.c0, 0), __shfl_sync(0xffffffffu, mine.row, 0)};
        const SharedParts own{__shfl_sync(0xffffffffu, mine.n, 16), __shfl_sync(0xffffffffu, mine.c0, 16), __shfl_sync(0xffffffffu, mine.row, 16)};
        const int n = pre.n + own.n;
        // part i: where its o lies, and its m and l
        const auto find = [&](int i, const float** o, const float** ml, int* to_l) {
            const bool first = i < pre.n;
            const SharedParts s = first ? pre : own;
            const SharedLaunch& at = first ? p.prefix : p.own;
            if (s.n == 1) {
                const int64_t cell = ((int64_t)(first ? 0 : 1) * p.T + t) * p.h_q + head * p.group + r;
                *o = p.row_o + cell * D;
                *ml = reinterpret_cast<const float*>(p.row_ml + cell);
                *to_l = 1;
                return;
            }
            const int k = first ? i : i - pre.n, block_rows = 1 << (at.tiles ? p.log2_tile_rows : 3);
            const float* slot = at.partial + (int64_t)(2 * (s.c0 + k) + (k == 0 ? 1 : 0)) * (block_rows * (D + 2));
            *o = slot + s.row * D;
            *ml = slot + block_rows * D + s.row;
            *to_l = block_rows;
        };
        for (int at = 0; at < n; at += 32) {                         // 32 parts at a time, a lane each; m, and what it scales, follow
            const float *o = nullptr, *ml = nullptr;
            int to_l = 0;
            float m_part = -INFINITY, l_part = 0.f;
            if (at + lane < n) {
                find(at + lane, &o, &ml, &to_l);
                m_part = ml[0];
                l_part = ml[to_l];
            }
            float top = m_part;
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
            top = fmaxf(top, m);
            const float back = exp2_fast(m - top), f = exp2_fast(m_part - top);
            m = top;
            l = l * back + l_part * f;
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] *= back;
            const int here = min(32, n - at);
#pragma unroll (V == 8 ? 4 : 8)
            for (int j = sub; j < here; j += W) {
                const float* from = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(o), j)) + V * lane;
                const float fj = __shfl_sync(0xffffffffu, f, j);
                float y[V];
                if constexpr (V == 2) *reinterpret_cast<float2*>(y) = *reinterpret_cast<const float2*>(from);
                else
#pragma unroll
                    for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(y + e) = *reinterpret_cast<const float4*>(from + e);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = fmaf(y[e], fj, acc[e]);
            }
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);   // (each of the W warps has it whole)
    }
    if (W > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) sums[warp][e * 32 + lane] = acc[e];
        __syncthreads();
        if (sub == 0)
#pragma unroll
            for (int w = 1; w < W; ++w)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += sums[warp + w][e * 32 + lane];
    }
    if (sub == 0 && r < p.group) {
        const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
        __half* to = p.out + (int64_t)t * p.out_ld + (int64_t)(head * p.group + r) * D + V * lane;
#pragma unroll
        for (int e = 0; e < V; e += 2) *reinterpret_cast<__half2*>(to + e) = __floats2half2_rn(acc[e] * inv, acc[e + 1] * inv);
    }
}

}  // namespace ql
