// Attention of few query rows over the paged 4-bit cache of paged.cuh: a generated token of every sequence, or a few.
//
//   o[i, h] = sum_j w_j v_j / sum_j w_j,   w_j = exp(x_j - m),   x_j = scale q.k_j  (or cap tanh(scale q.k_j / cap)),   visible j only
//
// One pass over the cache with the running maximum and sum of the softmax.  A warp takes blocks of 16 tokens: the keys are the 16-row operand of
// mma.m16n8k16 (integers in fp16, exact; the scale of a token and group of 32 elements multiplies the group's fp32 sums), the 8 query rows its
// columns; the weights become the second product's operand by two 8 x 8 transpositions in registers, the values, unpacked and scaled to
// fp16(q s), its rows.  So no lane ever needs another's bytes but through the tensor core.
//
// Work: the segments (sequence, KV head, 8 query rows) of the batch, numbered through, each as long as its blocks and kAttnOverhead more
// (what a segment costs besides its blocks: an empty pipeline, the warps' meeting), are cut into one span of equal length per CTA, whatever the
// lengths: a ragged batch and a single long sequence load the SMs alike (64 sequences of 128 .. 8192 tokens, 194618 in all, 8 KV heads of 128:
// 81.7 us with spans of blocks alone, 72.3, 68.1, 64.1, 66.0 with 8, 16, 32, 48 more; of equal lengths 63).  The grid is the CTAs that
// run at once: two an SM, but one at d_h 256, where rings, queries and plan take more than half of an SM's shared memory (24 sequences of up to 7001, window 4096: 38.6 us with a grid for two,
// 31.9 for one, 29.5 with the registers of one), and at d_h 128 beyond about 1650 sequences.  The plan is made by every CTA
// from the lengths on the device (a scan), so a captured launch follows them.  A CTA's 8 warps take the blocks of a segment in turn, each
// through a ring of its own in shared memory that goes on from segment to segment (bulk copies, requested by the lane that looked up the page), and
// meet at the segment's end, when the first blocks of the next one are on their way.  A segment cut by a span's end leaves (m, l, o) in the
// workspace, which paged_combine_kernel joins in order.  Weights are fp16, w_j = exp(x_j - m) with m lying 2^7 (kWeightLift) below the largest score when it is set
// and raised only when a score passes it by 2^15: they use the range up to 2^15 of fp16's 2^16, and what vanishes from the products, weights below 2^-25, is below 2^-32 of the largest
// (at m = the largest score it was 2^-25 of it, and the weight of 100000 such tokens, which the fp32 sums of weights did count, was missing from the result).
//
// Bound: the instructions that unpack, not the memory.  About 430 warp instructions per block of 16 tokens and 128 elements give 4.5 TB/s of cache
// in the loop; 131071 tokens of one sequence take 43 us (151 MB, 23 us at the copy rate), of which 8 are the two launches' fixed part.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "dequant.cuh"
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace ql {

constexpr float kWeightLift = 7.f, kWeightRange = 15.f;                  // the largest weight is 2^7 when m is set, m is raised before one passes 2^15
constexpr float kMostScale = 1e15f;                                      // scores stay far above -1e30, what a row's m is before its first token (products of fp16 vectors are below 2e12)
constexpr int kAttnWarps = 8;
constexpr int kAttnCols = 8;
// The query rows per KV head that this kernel takes, 8 at a time; more go to paged_tiles.cuh, whose time does not depend on them (us, here and there, 16 sequences of 4096: 16 KV heads
// of 64, 40 rows 118 and 134, 48 rows 140 and 134, 64 rows 183 and 134; 8 of 128, 32 rows 78 and 87, 40 rows 94 and 88; 4 of 256, 16 rows 44 and 67, 24 rows 60 and 67, 32 rows 77 and 67).  The
// rule goes by the rows alone, for batches: of ONE long sequence this kernel would still take 40 to 64 rows faster (16384: 40 rows 35 and 47, 31 and 41, 30 and 48).
__host__ __device__ constexpr int attn_max_rows(int d) { return d == 64 ? 48 : d == 128 ? 32 : 24; }
constexpr int kAttnOverhead = 32;                                        // a segment without blocks, in blocks
constexpr int kAttnSpan = 16;                                            // the least span: two blocks per warp (4096 tokens, 8 KV heads: 11.1, 11.4, 10.6 us with 8, 16, 24; 512 tokens: 8.6, 9.2, 9.8; four of 1280: 11.2, 11.3, 12.0)
template <int D> struct AttnRing {
    static constexpr int kBlock = paged_block_bytes(D);
    static constexpr int kStages = D == 64 ? 6 : D == 128 ? 4 : 3;
    static constexpr int kRing = kAttnWarps * kStages * kBlock;
    static constexpr int kMergeStride = D + 4;                           // floats of a column in the warps' meeting
    static constexpr bool kMeetApart = D < 256;                          // a buffer of its own for it: the ring already has the next segment's blocks
    static constexpr int kMeet = kAttnWarps * kAttnCols * kMergeStride * 4;
    static constexpr int kBytes = kRing + (kMeetApart ? kMeet : 0);
    static_assert(kMeet <= kRing, "or the ring's memory");
};

__device__ __forceinline__ float exp2_fast(float x)                      // (2 ulp; subnormal results are zero)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float rcp_fast(float x)                       // (1 ulp; 0 of infinity)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float a0, float a1, float b, float c)                           // (a0 b + c, a1 b + c)
{
    float2 r;
    asm("{\n\t.reg .b64 a, b, c, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%5, %5};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a0), "f"(a1), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 r;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
// The soft cap of scores on a base-2 scale: cap log2(e) tanh(y), y = scale dot / cap.  One of two forms, chosen by the host:
// kCapPlain, caps up to 128: tanh(y) = 1 - 2 / (exp(2 y) + 1), whose rounding errors are of 1, so that a score is off by up to 6 * 2^-24 cap: below 2^-14 there, an eighth of what the
// fp16 weights are rounded by.  A higher cap would lose the scores in it (10^5: 2 % of a weight; 10^8: everything).
// kCapHigh: for |y| < 1/4 the score times the series tanh(y) / y = 1 - y^2 / 3 + 2 y^4 / 15 - 17 y^6 / 315 (the next term is below 2^-21 there), else the same exponential: all errors are of
// the score, which stays what it is as the cap grows.  Five more instructions a score: two prompts of 4096, 4 KV heads of 128, 184 us plain and 240 high; a token of 24 sequences of 4096 23.5 and 24.9.
enum AttnCap { kCapNone, kCapPlain, kCapHigh };
constexpr float kMostPlainCap = 128.f;
struct SoftCap {
    float in, out, linear, shrink;
    __device__ SoftCap(float scale, float cap) : in(cap > 0.f ? 2.f * 1.4426950408889634f * scale / cap : 0.f), out(cap * 1.4426950408889634f), linear(scale * 1.4426950408889634f), shrink(cap > 0.f ? scale / cap : 0.f) {}
    template <AttnCap CAP, int N> __device__ __forceinline__ void on(float* x) const   // (two scores to an instruction: the kernel of many rows waits for its instructions)
    {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            const float2 dot = make_float2(x[e], x[e + 1]), a = mul2(dot, make_float2(in, in)), b = add2(make_float2(exp2_fast(a.x), exp2_fast(a.y)), make_float2(1.f, 1.f));
            float2 r = fma2(rcp_fast(b.x), rcp_fast(b.y), -2.f * out, out);
            if (CAP == kCapHigh) {
                const float2 y = mul2(dot, make_float2(shrink, shrink)), z = mul2(y, y), s = mul2(dot, make_float2(linear, linear));
                const float2 c = add2(mul2(z, add2(mul2(z, fma2(z.x, z.y, -17.f / 315, 2.f / 15)), make_float2(-1.f / 3, -1.f / 3))), make_float2(1.f, 1.f)), t = mul2(s, c);
                if (fabsf(y.x) < 0.25f) r.x = t.x;
                if (fabsf(y.y) < 0.25f) r.y = t.y;
            }
            x[e] = r.x;
            x[e + 1] = r.y;
        }
    }
};

// What a call's segments are: kAttnAll, the tokens that a row sees (qlinear_paged_attention); kAttnListed, those of the pages listed for a row and KV head (.._selected), a segment per row; kAttnShared, the
// shared beginning of a group's sequences for all rows of the group, and what follows of each sequence (.._shared), as paged_shared.cuh planned them: no segment is a row's whole result there.
enum AttnKind { kAttnAll, kAttnListed, kAttnShared };

// A stretch of tokens that some rows see (kAttnShared): rows t0 .. of the call, row 0's position, tokens first .. end - 1 (first a multiple of 64) as far as a row's position goes.
struct AttnStretch {
    int32_t t0, rows, pos0, first, end, seq, blocks, row_blocks;         // blocks of 16 tokens, blocks of kAttnCols rows: of the kernel of few rows
};

struct PagedAttnParams {
    PagedBatch batch;
    const __half* q;             // row t, head h at q + t * q_ld + h * D
    __half* out;                 // the same with out_ld
    float* partial;              // [2 * gridDim.x][rows * D of o, rows of m, rows of l]; slot 1 of a CTA: the first part of a segment, slot 0: a later one
    int4* split;                 // per CTA: sequence (-1: none), KV head, row block of the segment that begins in its span and ends in another's, and the last CTA that holds a part
    int64_t q_ld, out_ld;
    int32_t h_q, group, max_q, row_blocks, window;
    float scale, softcap;        // (softcap 0: none; not so far from the scale that SoftCap's constants leave fp32)
    int32_t grid;
    // kAttnListed: columns of the page table [T, h_kv, budget]
    const int32_t* pages;
    int32_t budget;
    // kAttnShared: stretches v0 .. v1 - 1 are this launch's; the first n_groups are groups'; sums of their lengths; o, and m and l, of the rows of uncut segments [2][T][h_q]
    int32_t v0, v1, n_groups;
    const AttnStretch* stretches;
    const int32_t* lengths;
    float* row_o;
    float2* row_ml;
};
// Where the result of a row lies that an uncut segment of a stretch leaves.
__device__ __forceinline__ int64_t attn_row(const PagedAttnParams& p, int part, int t, int head, int in_group)
{
    return ((int64_t)part * p.batch.T + t) * p.h_q + head * p.group + in_group;
}
// Blocks of the pages listed for a row of sequence b.
__device__ __forceinline__ int listed_blocks(const PagedAttnParams& p, int b)
{
    const int len = p.batch.kv_len[b];
    return len <= 0 ? 0 : min(p.budget, ((len - 1) >> (p.batch.log2_blocks + 4)) + 1) << p.batch.log2_blocks;
}

// Blocks [*first, *first + n) of 16 tokens that any served row of sequence b sees.
__device__ __forceinline__ int attn_blocks(const PagedAttnParams& p, int b, int* first)
{
    int t0;
    const int rows = paged_rows(p.batch, b, &t0);
    const int len = p.batch.kv_len[b];
    const int64_t held = (int64_t)p.batch.table_width << (p.batch.log2_blocks + 4);
    const int end = (int)max(min((int64_t)len - rows + min(rows, p.max_q), held), (int64_t)0);   // (up to the last served row's token)
    *first = 0;
    if (min(rows, p.max_q) <= 0 || end <= 0) return 0;
    if (p.window > 0) *first = (int)max((int64_t)len - rows + 1 - p.window, (int64_t)0) >> 4;   // the first token that the first row sees
    return max(0, (int)(((unsigned)end + 15) >> 4) - *first);
}

__device__ __forceinline__ uint32_t move_matrix(uint32_t a)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}
// Sums over a scan of the sequences' lengths: pre[b] before sequence b (per head and row block).  Every thread takes part.
template <AttnKind KIND>
__device__ __forceinline__ void attn_scan(const PagedAttnParams& p, int* pre)
{
    __shared__ int warp_sum[kAttnWarps];
    const int B = p.batch.B, tid = threadIdx.x, per = (B + 255) / 256, lo = min(B, tid * per), hi = min(B, lo + per);
    int sum = 0, first;
    unsigned long long wide = 0;
    for (int b = lo; b < hi; ++b) {
        const int blocks = KIND == kAttnListed ? listed_blocks(p, b) : attn_blocks(p, b, &first);
        int n = blocks > 0 ? blocks + kAttnOverhead : 0;
        if (KIND == kAttnListed) {                                       // (a segment per row)
            const int rows = paged_rows(p.batch, b, &first);
            wide += (unsigned long long)n * rows;
            n *= rows;
        }
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
    if constexpr (KIND == kAttnListed)                                   // rows named more than once, against the rules, may add up beyond 32 bits: nothing is done for them
        if (__syncthreads_or(wide > INT32_MAX / (kAttnWarps * 32))) {
            __shared__ unsigned long long all;
            if (tid == 0) all = 0;
            __syncthreads();
            atomicAdd(&all, wide);
            __syncthreads();
            if (all > INT32_MAX)
                for (int b = tid; b <= B; b += kAttnWarps * 32) pre[b] = 0;
            __syncthreads();
        }
}

// What a CTA does of a segment: blocks first .. first + n - 1 of its sequence.
struct AttnSegment {
    int32_t head, row0, n_rows, t0, pos0, first, n, slot;                // rows of the sequence row0 .. (n_rows of it), row 0's token and position; slot -1: the whole segment
    int64_t table, next;                                                 // offset of the sequence's row of the page table; where the next segment begins in the numbering
};
struct ListedSegment : AttnSegment { int64_t list; };                    // offset of the row's list

template <int D, AttnCap CAP, AttnKind KIND = kAttnAll>
__global__ void __launch_bounds__(kAttnWarps * 32, D == 256 ? 1 : 2) paged_attention_kernel(const PagedAttnParams p)
{
    constexpr int NB = D / 64, kBlock = AttnRing<D>::kBlock, S = AttnRing<D>::kStages, kStride = AttnRing<D>::kMergeStride;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float meet_m[2][kAttnWarps][kAttnCols], meet_l[2][kAttnWarps][kAttnCols];
    __shared__ __align__(8) uint64_t bars[kAttnWarps * S];
    using Segment = std::conditional_t<KIND == kAttnListed, ListedSegment, AttnSegment>;
    __shared__ int where[KIND == kAttnListed ? kAttnWarps * S : 1];      // the block of the sequence in a stage of a ring, -1: none
    __shared__ Segment segs[4];                                      // in turn: the last one (slow warps still look at it), this, the next, the one after it
    __shared__ volatile uint32_t abort_flag[4];
    // (at d_h 256 the queries lie in shared memory, read for every block)
    constexpr bool kQueriesApart = D == 256;
    __shared__ __align__(16) uint4 queries[kQueriesApart ? 2 * NB * 32 : 1];
    int* pre = reinterpret_cast<int*>(smem + AttnRing<D>::kBytes);       // [B + 1]
    float* meet = reinterpret_cast<float*>(smem + (AttnRing<D>::kMeetApart ? AttnRing<D>::kRing : 0));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const uint32_t bar0 = smem_u32(bars) + warp * (S * 8), ring_u32 = smem_u32(smem) + warp * (S * kBlock);
    const uint8_t* ring = smem + warp * (S * kBlock);
    if (lane < S) mbar_init(bar0 + 8 * lane, 1);
    if (tid == 0) { abort_flag[0] = abort_flag[1] = 0; abort_flag[2] = abort_flag[3] = 1; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if constexpr (KIND == kAttnShared) {
        for (int v = tid; v <= p.v1 - p.v0; v += kAttnWarps * 32) pre[v] = p.lengths[p.v0 + v] - p.lengths[p.v0];
        __syncthreads();
    } else {
        attn_scan<KIND>(p, pre);
    }

    const int h_kv = p.batch.h_kv, per_head = KIND == kAttnShared ? h_kv : h_kv * p.row_blocks, n_seqs = KIND == kAttnShared ? p.v1 - p.v0 : p.batch.B;   // (a stretch's length has its row blocks in it)
    const int64_t total = (int64_t)pre[n_seqs] * per_head;
    const int64_t span = max((int64_t)kAttnSpan, (total + p.grid - 1) / p.grid);
    const int64_t w0 = (int64_t)blockIdx.x * span, w1 = min(total, w0 + span);
    if (KIND != kAttnShared && tid == 0) p.split[blockIdx.x] = make_int4(-1, 0, 0, 0);
    for (int b = blockIdx.x; KIND != kAttnShared && b < p.batch.B; b += p.grid) {   // rows of sequences that see nothing: zeros
        int t0;
        const int rows = min(paged_rows(p.batch, b, &t0), p.max_q);
        if (pre[b + 1] > pre[b]) continue;
        for (int64_t e = tid; e < (int64_t)rows * p.h_q * (D / 8); e += kAttnWarps * 32)
            *reinterpret_cast<uint4*>(p.out + (t0 + e / (p.h_q * (D / 8))) * p.out_ld + 8 * (e % (p.h_q * (D / 8)))) = make_uint4(0, 0, 0, 0);
    }
    // The first segment from place w of the numbering on of which this CTA has blocks (n 0: none).  (by the warp with the fewest blocks; every lane computes it)
    const auto describe = [&](int64_t w, Segment* to) {
        Segment s{};
        while (w < w1) {
            const int x = (int)(w / per_head);
            int lo = 0, hi = n_seqs;                                     // pre[lo] <= x < pre[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (pre[mid] <= x) lo = mid;
                else hi = mid;
            }
            const int b = lo;
            int length = pre[b + 1] - pre[b];
            AttnStretch v;
            if constexpr (KIND == kAttnListed) length = listed_blocks(p, b) + kAttnOverhead;
            if constexpr (KIND == kAttnShared) { v = p.stretches[p.v0 + b]; length = v.blocks + kAttnOverhead; }
            const int blocks = length - kAttnOverhead;
            const int64_t local = w - (int64_t)pre[b] * per_head;
            const int seg = (int)(local / length), ua = (int)(local - (int64_t)seg * length), ub = (int)min((int64_t)length, ua + (w1 - w));
            const int sa = max(ua - kAttnOverhead, 0), sb = max(ub - kAttnOverhead, 0);
            const int64_t begin = w - ua;
            w += ub - ua;
            if (sb <= sa) continue;
            s.n = sb - sa;
            const bool whole = sa == 0 && sb == blocks;
            s.slot = whole ? -1 : sa > 0 ? 0 : 1;
            if constexpr (KIND == kAttnShared) {
                s.head = seg / v.row_blocks;
                s.row0 = (seg - s.head * v.row_blocks) * kAttnCols;
                s.n_rows = v.rows * p.group;
                s.t0 = v.t0;
                s.pos0 = v.pos0;
                s.first = v.first / kPagedBlock + sa;
                s.table = v.seq * p.batch.table_ld;
                if (whole && p.v0 + b >= p.n_groups) s.slot = -2;        // (uncut segments of a group's beginning and of what follows leave their rows apart)
            } else {
                int first = 0;
                if (KIND == kAttnAll) attn_blocks(p, b, &first);
                const int rows_all = paged_rows(p.batch, b, &s.t0), row = KIND == kAttnListed ? seg / per_head : 0, in_row = seg - row * per_head;
                s.head = in_row / p.row_blocks;
                s.row0 = (in_row - s.head * p.row_blocks) * kAttnCols;
                s.n_rows = KIND == kAttnListed ? p.group : min(rows_all, p.max_q) * p.group;
                s.pos0 = p.batch.kv_len[b] - rows_all + row;
                s.t0 += row;
                s.first = first + sa;
                s.table = b * p.batch.table_ld;
                if constexpr (KIND == kAttnListed) s.list = ((int64_t)s.t0 * h_kv + s.head) * p.budget;
                if (sa == 0 && !whole && lane == 0) p.split[blockIdx.x] = make_int4(KIND == kAttnListed ? s.t0 : b, s.head, s.row0 / kAttnCols, (int)((begin + length - 1) / span));
            }
            break;
        }
        s.next = w;
        if (lane == 0) *to = s;
        return s.next;
    };
    __syncthreads();                                                     // (p.split)
    if (warp == kAttnWarps - 1) describe(w0, &segs[0]);
    __syncthreads();

    // Blocks warp, warp + 8, ... of a segment are this warp's; the ring goes on from segment to segment.  Their places are found 32 at a time: `src` in lane k is that of block k
    // of a window, page_next the page of a block of the window after it, and none_even, none_odd tell which blocks of an even or odd window have no page (none_after: of the next segment's first).
    const uint8_t* src = nullptr;
    int page_next = -1, stage = 0, parity = 0, to = 0;                   // the stage (and its phase) that is read next, the one that is filled next
    uint32_t none_even = 0, none_odd = 0, none_after = 0;
    int column_next = -1, block_at = -1;                                 // kAttnListed: the column listed for it, and the block of the sequence that lane k's is
    const auto mine_of = [&](const Segment& s) { return s.n > warp ? (s.n - warp + kAttnWarps - 1) / kAttnWarps : 0; };
    const auto look_up = [&](const Segment& s, int i) {                  // the page of block i + lane
        if constexpr (KIND == kAttnListed) {
            const int entry = (s.first + warp + (i + lane) * kAttnWarps) >> p.batch.log2_blocks;
            column_next = i + lane < mine_of(s) ? p.pages[s.list + entry] : -1;
            if (column_next >= min(p.batch.table_width, 1 << (27 - p.batch.log2_blocks))) column_next = -1;   // (tokens of 31 bits)
            page_next = column_next >= 0 ? p.batch.table[s.table + column_next] : -1;
            return;
        }
        const int at = (s.first + warp + (i + lane) * kAttnWarps) >> p.batch.log2_blocks;
        page_next = i + lane < mine_of(s) && at < p.batch.table_width ? p.batch.table[s.table + at] : -1;
    };
    const auto place = [&](const Segment& s, int i) {                // of block i + lane, from the page that has been looked up; which have none
        const bool ok = page_next >= 0 && page_next < p.batch.n_pages;
        const int u = s.first + warp + (i + lane) * kAttnWarps;
        if (KIND == kAttnListed) block_at = ok ? column_next << p.batch.log2_blocks | (u & ((1 << p.batch.log2_blocks) - 1)) : -1;
        src = p.batch.pool + ((((int64_t)(ok ? page_next : 0) * h_kv + s.head) << p.batch.log2_blocks) + (u & ((1 << p.batch.log2_blocks) - 1))) * kBlock;
        return ~__ballot_sync(0xffffffffu, ok);
    };
    const auto request = [&](int i) {                                    // (block i lies in the window of `src`)
        if (lane == (i & 31)) {
            if (KIND == kAttnListed) where[warp * S + to] = block_at;    // (seen by those who have waited for the stage)
            mbar_expect_tx(bar0 + 8 * to, kBlock);
            bulk_copy_g2s(ring_u32 + to * kBlock, src, kBlock, bar0 + 8 * to);
        }
        to = to + 1 == S ? 0 : to + 1;
    };
    int requested = 0;                                                   // blocks of the segment, and on into the next one
    const float mag = fabsf(p.scale), cc = CAP ? 1.f : fmaxf(mag * 1.4426950408889634f, 1e-30f), margin = kWeightRange / cc;   // weights exp2(cc (x - m)); (cc never 0: hidden scores are -infinity)
    const uint32_t sign = p.scale < 0.f ? 0x80008000u : 0u;
    const SoftCap cap(mag, p.softcap);

    uint32_t qf[kQueriesApart ? 1 : NB][2][4];
    const auto load_queries = [&](const Segment& s) {                // column g of the second operand
        const int r = s.row0 + g, i = r / p.group;
        const __half* from = p.q + (int64_t)(s.t0 + i) * p.q_ld + (int64_t)(s.head * p.group + r - i * p.group) * D + 8 * c;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (kQueriesApart && (2 * j + e) % kAttnWarps != warp) continue;
                uint4 u = r < s.n_rows ? *reinterpret_cast<const uint4*>(from + 64 * j + 32 * e) : make_uint4(0, 0, 0, 0);
                u.x ^= sign; u.y ^= sign; u.z ^= sign; u.w ^= sign;
                if (kQueriesApart) queries[(2 * j + e) * 32 + lane] = u;
                else { qf[j % (kQueriesApart ? 1 : NB)][e][0] = u.x; qf[j % (kQueriesApart ? 1 : NB)][e][1] = u.y; qf[j % (kQueriesApart ? 1 : NB)][e][2] = u.z; qf[j % (kQueriesApart ? 1 : NB)][e][3] = u.w; }
            }
    };

    look_up(segs[0], 0);
    if (segs[0].n > 0) load_queries(segs[0]);
    if (warp == kAttnWarps - 1) describe(segs[0].next, &segs[1]);
    __syncthreads();
    bool ok = true;
    int meeting = 0;
    for (int it = 0; segs[it].n > 0; it = (it + 1) & 3) {
        const Segment &s = segs[it], &nx = segs[(it + 1) & 3];
        const int n_mine = mine_of(s), n_next = mine_of(nx);
        if (n_mine == 0 || (requested > 0 && n_mine <= 32)) look_up(nx, 0);
        if (warp == kAttnWarps - 1) describe(nx.next, &segs[(it + 2) & 3]);
        // what this lane's two columns see: tokens (lowest, last]; every column of the tile sees the blocks `seen` on, n_seen of them
        int last[2], lowest[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = s.row0 + 2 * c + e, pos = s.pos0 + r / p.group;
            last[e] = r < s.n_rows ? pos : INT32_MAX;                    // (a column behind the last row: its result is not looked at)
            lowest[e] = p.window > 0 && r < s.n_rows ? pos - p.window : -1;
        }
        int all_last = min(last[0], last[1]), all_lowest = max(lowest[0], lowest[1]);
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            all_last = min(all_last, __shfl_xor_sync(0xffffffffu, all_last, o));
            all_lowest = max(all_lowest, __shfl_xor_sync(0xffffffffu, all_lowest, o));
        }
        const int seen = (all_lowest + 16) >> 4, n_seen = max(((int)min((int64_t)all_last + 1, (int64_t)INT32_MAX) >> 4) - seen, 0);

        float o[NB][4][4];
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][h][e] = 0.f;
        float m0 = -1e30f, m1 = -1e30f, l0 = 0.f, l1 = 0.f;
        int u = s.first + warp;
#pragma unroll 1
        for (int i = 0; i < n_mine; ++i, u += kAttnWarps) {
            fence_async_smem();                                          // (every lane's reads of the block before come before the copy over it)
            __syncwarp();
            while (requested < min(i + S, AttnRing<D>::kMeetApart ? n_mine + n_next : n_mine)) {
                const bool here = requested < n_mine;
                const int k = here ? requested : requested - n_mine;
                if ((k & 31) == 0) {
                    const Segment& of = here ? s : nx;
                    const uint32_t none = place(of, k);
                    if (!here) none_after = none;
                    else if (k & 32) none_odd = none;
                    else none_even = none;
                    if (k + 32 < (here ? n_mine : n_next)) look_up(of, k + 32);
                    else if (here) look_up(nx, 0);
                }
                request(k);
                ++requested;
            }
            if (!__all_sync(0xffffffffu, mbar_wait_hot(bar0 + 8 * stage, parity, abort_flag, 0xA00))) {
                ok = false;
                requested -= i;
                break;
            }
            const int block = KIND == kAttnListed ? where[warp * S + stage] : u;
            const bool no_page = KIND == kAttnListed ? block < 0 : (i & 32 ? none_odd : none_even) >> (i & 31) & 1;
            const uint8_t* blk = ring + stage * kBlock;
            if (++stage == S) { stage = 0; parity ^= 1; }

            // scores
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            uint32_t ks[2 * NB];                                         // scales: (token g, token g + 8) per group
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
                    uint4 q;
                    if (kQueriesApart) q = queries[(2 * j + e) * 32 + lane];
                    else q = make_uint4(qf[j % (kQueriesApart ? 1 : NB)][e][0], qf[j % (kQueriesApart ? 1 : NB)][e][1], qf[j % (kQueriesApart ? 1 : NB)][e][2], qf[j % (kQueriesApart ? 1 : NB)][e][3]);
                    mma_16816_zero(t, a0, q.x, q.y);
                    mma_16816_pure(t, a1, q.z, q.w);
                    const float2 sc = __half22float2(*reinterpret_cast<const __half2*>(&ks[2 * j + e]));
                    x[0] = fmaf(t[0], sc.x, x[0]); x[1] = fmaf(t[1], sc.x, x[1]);
                    x[2] = fmaf(t[2], sc.y, x[2]); x[3] = fmaf(t[3], sc.y, x[3]);
                }
            }
            if (CAP) cap.on<CAP, 4>(x);
            // hidden tokens (only blocks that some column does not see whole, or without a page)
            if ((uint32_t)(block - seen) >= (uint32_t)n_seen || no_page) {
                const int j0 = block * 16;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + g + 8 * (e >> 1);
                    if (j > last[e & 1] || j <= lowest[e & 1] || no_page) x[e] = -INFINITY;
                }
            }
            // m is raised when a weight would pass 2^15
            if (__any_sync(0xffffffffu, fmaxf(x[0], x[2]) - m0 > margin || fmaxf(x[1], x[3]) - m1 > margin)) {   // (differences: exact however large the scores are)
                float n0 = fmaxf(x[0], x[2]), n1 = fmaxf(x[1], x[3]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, d));
                    n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, d));
                }
                constexpr float kLift = kWeightLift / kWeightRange;
                n0 = fmaxf(fmaf(margin, -kLift, n0), m0); n1 = fmaxf(fmaf(margin, -kLift, n1), m1);
                const float f0 = exp2_fast((m0 - n0) * cc), f1 = exp2_fast((m1 - n1) * cc);
                m0 = n0; m1 = n1; l0 *= f0; l1 *= f1;
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int h = 0; h < 4; ++h) { o[j][h][0] *= f0; o[j][h][1] *= f1; o[j][h][2] *= f0; o[j][h][3] *= f1; }
            }
            x[0] = exp2_fast((x[0] - m0) * cc); x[1] = exp2_fast((x[1] - m1) * cc); x[2] = exp2_fast((x[2] - m0) * cc); x[3] = exp2_fast((x[3] - m1) * cc);
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
        if (ok) requested -= n_mine;
        // the warps meet: o of column col in meet[warp][col][*]
        float (*mm)[kAttnCols] = meet_m[meeting], (*ml)[kAttnCols] = meet_l[meeting];
        meeting ^= 1;
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        if (g == 0) {
            mm[warp][2 * c] = m0; mm[warp][2 * c + 1] = m1;
            ml[warp][2 * c] = l0; ml[warp][2 * c + 1] = l1;
        }
        __syncthreads();
        float M0 = -1e30f, M1 = -1e30f;
#pragma unroll
        for (int k = 0; k < kAttnWarps; ++k) { M0 = fmaxf(M0, mm[k][2 * c]); M1 = fmaxf(M1, mm[k][2 * c + 1]); }
        const float f0 = exp2_fast((m0 - M0) * cc), f1 = exp2_fast((m1 - M1) * cc);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            float* to = meet + (warp * kAttnCols + 2 * c) * kStride + 64 * j + 8 * g;
            *reinterpret_cast<float4*>(to) = make_float4(o[j][0][0] * f0, o[j][0][2] * f0, o[j][1][0] * f0, o[j][1][2] * f0);
            *reinterpret_cast<float4*>(to + 4) = make_float4(o[j][2][0] * f0, o[j][2][2] * f0, o[j][3][0] * f0, o[j][3][2] * f0);
            *reinterpret_cast<float4*>(to + kStride) = make_float4(o[j][0][1] * f1, o[j][0][3] * f1, o[j][1][1] * f1, o[j][1][3] * f1);
            *reinterpret_cast<float4*>(to + kStride + 4) = make_float4(o[j][2][1] * f1, o[j][2][3] * f1, o[j][3][1] * f1, o[j][3][3] * f1);
        }
        if (nx.n > 0) load_queries(nx);
        __syncthreads();
        float* part = p.partial + (int64_t)(2 * blockIdx.x + max(s.slot, 0)) * (kAttnCols * (D + 2));
        for (int e = tid * 4; e < kAttnCols * D; e += kAttnWarps * 32 * 4) {
            const int col = e / D, d = e - col * D, r = s.row0 + col;
            float top = -1e30f, l = 0.f;
#pragma unroll
            for (int k = 0; k < kAttnWarps; ++k) top = fmaxf(top, mm[k][col]);
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kAttnWarps; ++k) {
                const float4 v = *reinterpret_cast<const float4*>(meet + (k * kAttnCols + col) * kStride + d);
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                l += ml[k][col] * exp2_fast((mm[k][col] - top) * cc);
            }
            if (s.slot >= 0) {
                *reinterpret_cast<float4*>(part + e) = sum;
                if (d == 0) { part[kAttnCols * D + col] = top * cc; part[kAttnCols * D + kAttnCols + col] = l; }
            } else if (KIND == kAttnShared) {
                const int i = r / p.group;
                const int64_t row = attn_row(p, -1 - s.slot, s.t0 + i, s.head, r - i * p.group);
                if (r < s.n_rows) {
                    *reinterpret_cast<float4*>(p.row_o + row * D + d) = sum;
                    if (d == 0) p.row_ml[row] = make_float2(top * cc, l);
                }
            } else if (r < s.n_rows) {
                const float inv = l > 0.f || l != l ? 1.f / l : 0.f;     // (no visible token: zeros)
                const int i = r / p.group;
                const __half2 y[2] = {__floats2half2_rn(sum.x * inv, sum.y * inv), __floats2half2_rn(sum.z * inv, sum.w * inv)};
                *reinterpret_cast<uint2*>(p.out + (int64_t)(s.t0 + i) * p.out_ld + (int64_t)(s.head * p.group + r - i * p.group) * D + d) = *reinterpret_cast<const uint2*>(y);
            }
        }
        if (abort_flag[0]) {                                             // a wait ran out (every warp is past this segment's): the copies in flight land first
            for (; requested > 0; --requested) {
                mbar_wait(bar0 + 8 * stage, parity, abort_flag + 1, 0);
                if (++stage == S) { stage = 0; parity ^= 1; }
            }
            break;
        }
        if (!AttnRing<D>::kMeetApart) {                                  // (the sums have been read: the ring's memory is free)
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncthreads();
        }
        none_even = none_after;
    }
}

// Joins the parts of the segment that begins in a CTA's span and ends in another's, in a fixed order: CTA blockIdx.x's, 8 / W x R of its rows
// per CTA.  W warps share a row's parts, 8 of them in flight each: one long sequence is many parts of few segments, and reading them one after
// the other took as long as a fifth of the pass (131071 tokens, 8 KV heads of 128, 37 parts each: 52.8 -> 42.8 us for the call).
template <int D, int ROWS, int R, int W, AttnKind KIND = kAttnAll>
__global__ void __launch_bounds__(256) paged_combine_kernel(const PagedAttnParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    static_assert(W == 1 || R == 1, "");
    constexpr int V = D / 32, kAhead = 8 / R;                            // values of a lane; parts whose loads are in flight
    constexpr int64_t kStride = ROWS * (D + 2);
    __shared__ __align__(16) float sums[W > 1 ? 8 : 1][D];
    __shared__ float sums_l[W > 1 ? 8 : 1];
    const int4 split = p.split[blockIdx.x];
    if (split.x < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = (blockIdx.y * (8 / W) + warp / W) * R, sub = warp % W;
    const int c0 = blockIdx.x, parts = split.w - c0 + 1;
    int t0;
    int n_rows = p.group;
    if (KIND == kAttnListed) t0 = split.x;                               // (a row's segment)
    else n_rows = min(paged_rows(p.batch, split.x, &t0), p.max_q) * p.group;
    if (split.z * ROWS + blockIdx.y * (8 / W) * R >= n_rows) return;     // (the whole CTA; ROWS and the partial results hold the rows behind the last one)
    const auto part_of = [&](int c) { return p.partial + (2 * (c0 + c) + (c == 0 ? 1 : 0)) * kStride; };
    float m[R], l[R], acc[R][V];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        m[k] = -1e30f;
        l[k] = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[k][e] = 0.f;
    }
    for (int c = lane; c < parts; c += 32)
#pragma unroll
        for (int k = 0; k < R; ++k) m[k] = fmaxf(m[k], part_of(c)[ROWS * D + row + k]);
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m[k] = fmaxf(m[k], __shfl_xor_sync(0xffffffffu, m[k], o));
    for (int at = sub; at < parts; at += 32 * W) {                       // 32 parts' weights side by side, then their values
        float f[R];
        const int mine = at + lane * W, n = min(32, (parts - at + W - 1) / W);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const float* part = part_of(min(mine, parts - 1)) + ROWS * D + row + k;
            f[k] = mine < parts ? exp2_fast(part[0] - m[k]) : 0.f;
            l[k] += mine < parts ? part[ROWS] * f[k] : 0.f;
        }
#pragma unroll kAhead
        for (int j = 0; j < n; ++j) {
            const float* part = part_of(at + j * W) + row * D + V * lane;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float fj = __shfl_sync(0xffffffffu, f[k], j);
                float y[V];
                if constexpr (V == 2) *reinterpret_cast<float2*>(y) = *reinterpret_cast<const float2*>(part + k * D);
                else
#pragma unroll
                    for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(y + e) = *reinterpret_cast<const float4*>(part + k * D + e);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[k][e] = fmaf(y[e], fj, acc[k][e]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l[k] += __shfl_xor_sync(0xffffffffu, l[k], o);
    if constexpr (W > 1) {
#pragma unroll
        for (int e = 0; e < V; ++e) sums[warp][e * 32 + lane] = acc[0][e];
        if (lane == 0) sums_l[warp] = l[0];
        __syncthreads();
        if (sub > 0) return;
#pragma unroll
        for (int w = 1; w < W; ++w) {
            l[0] += sums_l[warp + w];
#pragma unroll
            for (int e = 0; e < V; ++e) acc[0][e] += sums[warp + w][e * 32 + lane];
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
