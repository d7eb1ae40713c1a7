// Attention of few query rows over the paged 4-bit cache of paged.cuh: a generated token of every sequence, or a few.
//
//   o[i, h] = sum_j w_j v_j / sum_j w_j,   w_j = exp(x_j - m),   x_j = scale q.k_j  (or cap tanh(scale q.k_j / cap)),   visible j only
//
// One pass over the cache with the running maximum and sum of the softmax.  A warp takes blocks of 16 tokens: the keys are the 16-row operand of
// mma.m16n8k16 (integers in fp16, exact; the scale of a token and group of 32 elements multiplies the group's fp32 sums), the 8 query rows its
// columns; the weights become the second product's operand by two 8 x 8 transpositions in registers, the values, unpacked and scaled to
// fp16(q s), its rows.  So no lane ever needs another's bytes but through the tensor core.
//
// Work: the blocks of all (sequence, KV head, 8 query rows) segments, numbered through, are cut into one span of equal length per CTA, whatever the
// lengths: a ragged batch and a single long sequence load the SMs alike.  The plan is made by every CTA from the lengths on the device
// (a scan), so a captured launch follows them.  A CTA's 8 warps take the blocks of a segment in turn, each through a ring of its own in shared
// memory (cp.async), and meet at the segment's end; a segment cut by a span's end leaves (m, l, o) in the workspace, which paged_combine_kernel
// joins in order.  Weights are fp16 relative to a maximum that is raised only when it is passed by 2^8 (sums are fp32; at most 2^8 of
// 2^16 are used).
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dequant.cuh"
#include "paged.cuh"

namespace ql {

constexpr int kAttnWarps = 8;
constexpr int kAttnCols = 8;
constexpr int kAttnMaxRows = 32;                                         // query rows per KV head that this kernel takes (8 at a time); more: paged_tiles.cuh
template <int D> struct AttnRing {
    static constexpr int kBlock = paged_block_bytes(D);
    static constexpr int kStages = D == 64 ? 6 : D == 128 ? 4 : 3;
    static constexpr int kBytes = kAttnWarps * kStages * kBlock;
    static constexpr int kMergeStride = D + 4;                           // floats of a column in the warps' meeting (the ring's memory)
    static_assert(kAttnWarps * kAttnCols * kMergeStride * 4 <= kBytes, "the warps meet in the ring's memory");
};

struct PagedAttnParams {
    PagedBatch batch;
    const __half* q;             // row t, head h at q + t * q_ld + h * D
    __half* out;                 // the same with out_ld
    float* partial;              // [2 * gridDim.x][rows * D of o, rows of m, rows of l]; slot 1 of a CTA: the first part of a segment, slot 0: a later one
    int4* split;                 // per CTA: sequence (-1: none), KV head, row block of the segment that begins in its span and ends in another's, and the last CTA that holds a part
    int64_t q_ld, out_ld;
    int32_t h_q, group, max_q, row_blocks, window;
    float scale, softcap;        // (softcap 0: none)
    int32_t grid;
};

// Blocks [*first, *first + n) of 16 tokens that any row of sequence b sees.
__device__ __forceinline__ int attn_blocks(const PagedAttnParams& p, int b, int* first)
{
    int t0;
    const int rows = paged_rows(p.batch, b, &t0);
    const int len = p.batch.kv_len[b];
    const int64_t held = (int64_t)p.batch.table_width << (p.batch.log2_blocks + 4);
    const int end = (int)min((int64_t)len, held);
    *first = 0;
    if (min(rows, p.max_q) <= 0 || end <= 0) return 0;
    if (p.window > 0) *first = (int)max((int64_t)len - rows + 1 - p.window, (int64_t)0) >> 4;   // the first token that the first row sees
    return max(0, ((end + 15) >> 4) - *first);
}

__device__ __forceinline__ uint32_t move_matrix(uint32_t a)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ float exp2_fast(float x)                      // (2 ulp; subnormal results are zero)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The score of a key on a base-2 scale, after the soft cap.  tanh(y) = 1 - 2 / (exp(2 y) + 1).
template <bool CAP>
__device__ __forceinline__ float attn_score(float dot, float scale, float softcap)
{
    constexpr float kLog2e = 1.4426950408889634f;
    if (!CAP) return dot * (scale * kLog2e);
    return softcap * kLog2e * (1.f - __fdividef(2.f, exp2_fast(2.f * kLog2e * fminf(dot * scale / softcap, 40.f)) + 1.f));
}

// Sums over a scan of the sequences' block counts: pre[b] blocks before sequence b (per head and row block).  Every thread takes part.
__device__ __forceinline__ void attn_scan(const PagedAttnParams& p, int* pre)
{
    __shared__ int warp_sum[kAttnWarps];
    const int B = p.batch.B, tid = threadIdx.x, per = (B + 255) / 256, lo = min(B, tid * per), hi = min(B, lo + per);
    int sum = 0, first;
    for (int b = lo; b < hi; ++b) {
        const int n = attn_blocks(p, b, &first);
        pre[b + 1] = n;
        sum += n;
    }
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, run, o);
        if ((tid & 31) >= o) run += v;
    }
    if ((tid & 31) == 31) warp_sum[tid >> 5] = run;
    __syncthreads();
    run -= sum;
    for (int w = 0; w < (tid >> 5); ++w) run += warp_sum[w];
    for (int b = lo; b < hi; ++b) { run += pre[b + 1]; pre[b + 1] = run; }
    if (tid == 0) pre[0] = 0;
    __syncthreads();
}

template <int D, bool CAP>
__global__ void __launch_bounds__(kAttnWarps * 32, 2) paged_attention_kernel(const PagedAttnParams p)
{
    constexpr int NB = D / 64, kBlock = AttnRing<D>::kBlock, S = AttnRing<D>::kStages, kStride = AttnRing<D>::kMergeStride;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float meet_m[kAttnWarps][kAttnCols], meet_l[kAttnWarps][kAttnCols];
    int* pre = reinterpret_cast<int*>(smem + AttnRing<D>::kBytes);       // [B + 1]
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    attn_scan(p, pre);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int h_kv = p.batch.h_kv, segs = h_kv * p.row_blocks;
    const int64_t total = (int64_t)pre[p.batch.B] * segs;
    const int64_t span = max((int64_t)kAttnWarps, (total + p.grid - 1) / p.grid);
    const int64_t w0 = (int64_t)blockIdx.x * span, w1 = min(total, w0 + span);
    uint8_t* ring = smem + warp * (S * kBlock);
    const uint32_t ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);
    if (tid == 0) p.split[blockIdx.x] = make_int4(-1, 0, 0, 0);
    for (int b = blockIdx.x; b < p.batch.B; b += p.grid) {               // rows of sequences that see nothing: zeros
        int t0;
        const int rows = min(paged_rows(p.batch, b, &t0), p.max_q);
        if (pre[b + 1] > pre[b]) continue;
        for (int64_t e = tid; e < (int64_t)rows * p.h_q * (D / 8); e += kAttnWarps * 32)
            *reinterpret_cast<uint4*>(p.out + (t0 + e / (p.h_q * (D / 8))) * p.out_ld + 8 * (e % (p.h_q * (D / 8)))) = make_uint4(0, 0, 0, 0);
    }

    for (int64_t w = w0; w < w1;) {
        // the segment (sequence, KV head, 8 rows) and the part [ua, ub) of its blocks
        int b;
        {
            const int x = (int)(w / segs);
            int lo = 0, hi = p.batch.B;                                  // pre[lo] <= x < pre[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (pre[mid] <= x) lo = mid;
                else hi = mid;
            }
            b = lo;
        }
        const int blocks = pre[b + 1] - pre[b];
        const int64_t local = w - (int64_t)pre[b] * segs;
        const int seg = (int)(local / blocks), ua = (int)(local - (int64_t)seg * blocks), ub = (int)min((int64_t)blocks, ua + (w1 - w));
        const int head = seg / p.row_blocks, r0 = (seg - head * p.row_blocks) * kAttnCols;
        int first_block, t0;
        attn_blocks(p, b, &first_block);
        const int rows_all = paged_rows(p.batch, b, &t0), n_rows = min(rows_all, p.max_q) * p.group;
        const int len = p.batch.kv_len[b];
        const int32_t* table = p.batch.table + b * p.batch.table_ld;

        // the queries: column g of the second operand
        uint32_t qf[NB][2][4];
        {
            const int r = r0 + g, i = r / p.group;
            const __half* src = p.q + (int64_t)(t0 + i) * p.q_ld + (int64_t)(head * p.group + r - i * p.group) * D + 8 * c;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint4 u = r < n_rows ? *reinterpret_cast<const uint4*>(src + 64 * j + 32 * e) : make_uint4(0, 0, 0, 0);
                    qf[j][e][0] = u.x; qf[j][e][1] = u.y; qf[j][e][2] = u.z; qf[j][e][3] = u.w;
                }
        }
        // what this lane's two columns see: tokens (lowest, last]
        int last[2], lowest[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = r0 + 2 * c + e, pos = len - rows_all + r / p.group;
            last[e] = r < n_rows ? pos : -1;
            lowest[e] = p.window > 0 ? pos - p.window : -1;
        }
        int all_last = min(last[0], last[1]), all_lowest = max(lowest[0], lowest[1]);      // every column of the tile sees the tokens between
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            all_last = min(all_last, __shfl_xor_sync(0xffffffffu, all_last, o));
            all_lowest = max(all_lowest, __shfl_xor_sync(0xffffffffu, all_lowest, o));
        }

        float o[NB][4][4];
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][h][e] = 0.f;
        float m0 = -1e30f, m1 = -1e30f, l0 = 0.f, l1 = 0.f;

        // this warp's blocks ua + warp, + 8, ...: their pages are looked up 32 at a time
        const int n_mine = ub - ua > warp ? (ub - ua - warp + kAttnWarps - 1) / kAttnWarps : 0;
        const int u_first = first_block + ua + warp;
        int page = -1, page_next = -1;
        auto look_up = [&](int i) {                                      // the page of block i + lane of this warp's
            const int at = (u_first + (i + lane) * kAttnWarps) >> p.batch.log2_blocks;
            const int pg = i + lane < n_mine && at < p.batch.table_width ? table[at] : -1;
            return pg < p.batch.n_pages ? pg : -1;
        };
        page_next = look_up(0);
        // requests block i (a commit group in any case)
        auto request = [&](int i) {
            if ((i & 31) == 0) { page = page_next; page_next = look_up(i + 32); }
            const int pg = __shfl_sync(0xffffffffu, page, i & 31);
            if (i < n_mine) {
                const int u = u_first + i * kAttnWarps;
                const uint8_t* src = p.batch.pool + ((((int64_t)max(pg, 0) * h_kv + head) << p.batch.log2_blocks) + (u & ((1 << p.batch.log2_blocks) - 1))) * kBlock;
                const uint32_t dst = ring_u32 + (i % S) * kBlock;
#pragma unroll
                for (int k = 0; k < (kBlock + 511) / 512; ++k)
                    if ((k + 1) * 512 <= kBlock || k * 512 + lane * 16 < kBlock) cp_async16(dst + k * 512 + lane * 16, src + k * 512 + lane * 16);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            return pg;
        };
        int pages_ok[S];                                                 // (of the blocks in the ring: whether the table gave them a page)
#pragma unroll
        for (int i = 0; i < S - 1; ++i) pages_ok[i] = request(i);

        for (int i0 = 0; i0 < n_mine; i0 += S) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int i = i0 + s;
                if (i >= n_mine) break;
                asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
                __syncwarp();                                            // (this block has arrived for every lane, and no lane still reads the one before)
                pages_ok[(s + S - 1) % S] = request(i + S - 1);
                const uint8_t* blk = ring + s * kBlock;
                const int u = u_first + i * kAttnWarps;

                // scores
                float x[4] = {0.f, 0.f, 0.f, 0.f};
                uint32_t ks[2 * NB];                                     // (token g, token g + 8) per group
#pragma unroll
                for (int e = 0; e < NB; ++e)
                    *reinterpret_cast<uint2*>(ks + 2 * e) = *reinterpret_cast<const uint2*>(blk + paged_k_scales(D) + g * (8 * NB) + 8 * e);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const uint4 kw = *reinterpret_cast<const uint4*>(blk + 512 * j + 16 * lane);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t lo[4], hi[4];
                        unpack_int4_word(e ? kw.y : kw.x, lo);
                        unpack_int4_word(e ? kw.w : kw.z, hi);
                        float t[4];
                        const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
                        mma_16816_zero(t, a0, qf[j][e][0], qf[j][e][1]);
                        mma_16816_pure(t, a1, qf[j][e][2], qf[j][e][3]);
                        const float2 sc = __half22float2(*reinterpret_cast<const __half2*>(&ks[2 * j + e]));
                        x[0] = fmaf(t[0], sc.x, x[0]); x[1] = fmaf(t[1], sc.x, x[1]);
                        x[2] = fmaf(t[2], sc.y, x[2]); x[3] = fmaf(t[3], sc.y, x[3]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = attn_score<CAP>(x[e], p.scale, p.softcap);
                // hidden tokens (only blocks that some column does not see whole, or without a page)
                const int j0 = u * 16;
                if (j0 + 15 > all_last || j0 <= all_lowest || pages_ok[s] < 0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = j0 + g + 8 * (e >> 1);
                        if (j > last[e & 1] || j <= lowest[e & 1] || pages_ok[s] < 0) x[e] = -INFINITY;
                    }
                }
                // the maximum is raised when it is passed by 2^8
                if (__any_sync(0xffffffffu, fmaxf(x[0], x[2]) > m0 + 8.f || fmaxf(x[1], x[3]) > m1 + 8.f)) {
                    float n0 = fmaxf(x[0], x[2]), n1 = fmaxf(x[1], x[3]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, d));
                        n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, d));
                    }
                    n0 = fmaxf(n0, m0); n1 = fmaxf(n1, m1);
                    const float f0 = exp2_fast(m0 - n0), f1 = exp2_fast(m1 - n1);
                    m0 = n0; m1 = n1; l0 *= f0; l1 *= f1;
#pragma unroll
                    for (int j = 0; j < NB; ++j)
#pragma unroll
                        for (int h = 0; h < 4; ++h) { o[j][h][0] *= f0; o[j][h][1] *= f1; o[j][h][2] *= f0; o[j][h][3] *= f1; }
                }
                x[0] = exp2_fast(x[0] - m0); x[1] = exp2_fast(x[1] - m1); x[2] = exp2_fast(x[2] - m0); x[3] = exp2_fast(x[3] - m1);
                l0 += x[0] + x[2];
                l1 += x[1] + x[3];
                const __half2 p01 = __floats2half2_rn(x[0], x[1]), p23 = __floats2half2_rn(x[2], x[3]);
                const uint32_t b0 = move_matrix(*reinterpret_cast<const uint32_t*>(&p01)), b1 = move_matrix(*reinterpret_cast<const uint32_t*>(&p23));

                // values
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const uint4 vw = *reinterpret_cast<const uint4*>(blk + paged_v_data(D) + 512 * j + 16 * lane);
                    const uint2 vs = *reinterpret_cast<const uint2*>(blk + paged_v_scales(D) + (2 * j + (g >> 2)) * 32 + 8 * c);
                    uint32_t lo01[4], hi01[4], lo23[4], hi23[4];
                    unpack_int4_word(__byte_perm(vw.x, vw.y, 0x5410), lo01);
                    unpack_int4_word(__byte_perm(vw.x, vw.y, 0x7632), hi01);
                    unpack_int4_word(__byte_perm(vw.z, vw.w, 0x5410), lo23);
                    unpack_int4_word(__byte_perm(vw.z, vw.w, 0x7632), hi23);
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const uint32_t a[4] = {h2_mul(lo01[h], vs.x), h2_mul(hi01[h], vs.x), h2_mul(lo23[h], vs.y), h2_mul(hi23[h], vs.y)};
                        mma_16816_pure(o[j][h], a, b0, b1);
                    }
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");

        // the warps meet: o of column col in meet[warp][col][*], in the ring's memory
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        if (g == 0) {
            meet_m[warp][2 * c] = m0; meet_m[warp][2 * c + 1] = m1;
            meet_l[warp][2 * c] = l0; meet_l[warp][2 * c + 1] = l1;
        }
        __syncthreads();
        float M0 = -1e30f, M1 = -1e30f;
#pragma unroll
        for (int k = 0; k < kAttnWarps; ++k) { M0 = fmaxf(M0, meet_m[k][2 * c]); M1 = fmaxf(M1, meet_m[k][2 * c + 1]); }
        const float f0 = exp2_fast(m0 - M0), f1 = exp2_fast(m1 - M1);
        float* meet = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            float* to = meet + (warp * kAttnCols + 2 * c) * kStride + 64 * j + 8 * g;
            *reinterpret_cast<float4*>(to) = make_float4(o[j][0][0] * f0, o[j][0][2] * f0, o[j][1][0] * f0, o[j][1][2] * f0);
            *reinterpret_cast<float4*>(to + 4) = make_float4(o[j][2][0] * f0, o[j][2][2] * f0, o[j][3][0] * f0, o[j][3][2] * f0);
            *reinterpret_cast<float4*>(to + kStride) = make_float4(o[j][0][1] * f1, o[j][0][3] * f1, o[j][1][1] * f1, o[j][1][3] * f1);
            *reinterpret_cast<float4*>(to + kStride + 4) = make_float4(o[j][2][1] * f1, o[j][2][3] * f1, o[j][3][1] * f1, o[j][3][3] * f1);
        }
        __syncthreads();
        const bool whole = ua == 0 && ub == blocks;
        float* part = p.partial + (int64_t)(2 * blockIdx.x + (ua > 0 ? 0 : 1)) * (kAttnCols * (D + 2));
        for (int e = tid * 4; e < kAttnCols * D; e += kAttnWarps * 32 * 4) {
            const int col = e / D, d = e - col * D, r = r0 + col;
            float mm = -1e30f, l = 0.f;
#pragma unroll
            for (int k = 0; k < kAttnWarps; ++k) mm = fmaxf(mm, meet_m[k][col]);
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kAttnWarps; ++k) {
                const float4 v = *reinterpret_cast<const float4*>(meet + (k * kAttnCols + col) * kStride + d);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
                l += meet_l[k][col] * exp2_fast(meet_m[k][col] - mm);
            }
            if (!whole) {
                *reinterpret_cast<float4*>(part + e) = s;
                if (d == 0) { part[kAttnCols * D + col] = mm; part[kAttnCols * D + kAttnCols + col] = l; }
            } else if (r < n_rows) {
                const float inv = l > 0.f || l != l ? 1.f / l : 0.f;     // (no visible token: zeros)
                const int i = r / p.group;
                const __half2 y[2] = {__floats2half2_rn(s.x * inv, s.y * inv), __floats2half2_rn(s.z * inv, s.w * inv)};
                *reinterpret_cast<uint2*>(p.out + (int64_t)(t0 + i) * p.out_ld + (int64_t)(head * p.group + r - i * p.group) * D + d) = *reinterpret_cast<const uint2*>(y);
            }
        }
        if (tid == 0 && ua == 0 && !whole) p.split[blockIdx.x] = make_int4(b, head, seg - head * p.row_blocks, (int)((w + blocks - 1) / span));
        w += ub - ua;
        __syncthreads();                                                 // (the ring is free again)
    }
}

// Joins the parts of the segment that begins in a CTA's span and ends in another's, in order: CTA blockIdx.x's, ROWS / gridDim.y of its rows, R at a time per warp.
template <int D, int ROWS, int R>
__global__ void __launch_bounds__(256) paged_combine_kernel(const PagedAttnParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int V = D / 32;                                            // values of a lane
    constexpr int64_t kStride = ROWS * (D + 2);
    const int4 split = p.split[blockIdx.x];
    if (split.x < 0) return;
    const int row = (blockIdx.y * 8 + (threadIdx.x >> 5)) * R, lane = threadIdx.x & 31, c0 = blockIdx.x, c1 = split.w;
    int t0;
    const int n_rows = min(paged_rows(p.batch, split.x, &t0), p.max_q) * p.group;
    if (split.z * ROWS + row >= n_rows) return;
    const auto part_of = [&](int c) { return p.partial + (2 * c + (c == c0 ? 1 : 0)) * kStride; };
    float m[R], l[R], acc[R][V];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        m[k] = -1e30f;
        l[k] = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[k][e] = 0.f;
    }
    for (int c = c0 + lane; c <= c1; c += 32)
#pragma unroll
        for (int k = 0; k < R; ++k) m[k] = fmaxf(m[k], part_of(c)[ROWS * D + row + k]);
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m[k] = fmaxf(m[k], __shfl_xor_sync(0xffffffffu, m[k], o));
#pragma unroll 2
    for (int c = c0; c <= c1; ++c) {
        const float* part = part_of(c);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const float f = exp2_fast(part[ROWS * D + row + k] - m[k]);
            l[k] += part[ROWS * D + ROWS + row + k] * f;
#pragma unroll
            for (int e = 0; e < V; ++e) acc[k][e] = fmaf(part[(row + k) * D + V * lane + e], f, acc[k][e]);
        }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int r = split.z * ROWS + row + k, i = r / p.group;
        if (r >= n_rows) break;
        const float inv = l[k] > 0.f || l[k] != l[k] ? 1.f / l[k] : 0.f;
        __half* to = p.out + (int64_t)(t0 + i) * p.out_ld + (int64_t)(split.y * p.group + r - i * p.group) * D + V * lane;
#pragma unroll
        for (int e = 0; e < V; e += 2) *reinterpret_cast<__half2*>(to + e) = __floats2half2_rn(acc[k][e] * inv, acc[k][e + 1] * inv);
    }
}

}  // namespace ql
