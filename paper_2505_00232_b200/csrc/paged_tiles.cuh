// Attention of many query rows over the paged 4-bit cache of paged.cuh (prompts, chunks of them): the same operator as paged_attention.cuh, with the
// products on the 5th-generation tensor cores.
//
// A CTA works on a segment: 256 query rows (row = token * group + head of the group; 128 rows at d_h 256) of one KV head, and steps through the keys that any of
// them sees, 64 at a time.  Per step and tile of 128 rows:
//     S = Q K^T      tcgen05.mma, both operands in shared memory, S in tensor memory (fp32)
//     P = exp2(S c - m) as fp16, written over S in tensor memory by the softmax warps, a thread per row
//     O += P V       tcgen05.mma with P from tensor memory, O in tensor memory (fp32)
// so the scores never leave the SM and no thread needs another's row.  A tile has two buffers of S: the scores of the next step are computed while the softmax has
// the last ones, which never waits for the tensor core then (steps of 128 keys with one buffer per tile: 1073 TFLOP/s, a chunk of 4096 at 16384; the two tiles ran in
// step, softmax and products in turn).  The reference m of a row's weights is raised, and O rescaled, only when a weight would pass 2^15 (as in paged_attention.cuh).  Keys and values are unpacked from the cache's integers by warps of their own
// to fp16(q s), which go to shared memory in the operands' swizzled layout: K as rows of elements, V as rows of elements too, read transposed.
//
// Warps 0-3, 4-7: softmax of the two tiles (at d_h 256 there is one); warps 8-15: unpack; warps 16 and 17 issue the two products; warp 18 looks up the pages and
// requests the blocks of 16 tokens (bulk copies to a ring of raw steps in shared memory), so that nothing else waits for global memory between two
// segments but the softmax warps for the next queries, which they have copied (without passing through registers) while the last product runs.
// Bound: the softmax (64 exponentials, conversions and a maximum per row and step) and the shared memory's ports; a chunk of 4096 at 16384 runs at 1090 TFLOP/s.
//
// Work: the segments of the whole batch, numbered through, each as long as its steps and kTileOverhead more (queries in, rows out, an empty pipeline), in one span of
// equal length per CTA, as in paged_attention.cuh; a segment cut by a span's end leaves its rows' (m, l, O) in the workspace for paged_combine_kernel.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dequant.cuh"
#include "paged.cuh"
#include "paged_attention.cuh"
#include "sm100_ptx.cuh"

namespace ql {

template <int D> struct TileShape {
    static constexpr int NT = D == 256 ? 1 : 2;                          // tiles of 128 rows
    static constexpr int N = 64;                                         // keys of a step (a bit each of 64 in the softmax)
    static constexpr int kSlots = D == 256 ? 3 : D == 128 ? 6 : 8;       // operands in shared memory: K and V of the steps in turn
    static constexpr int kRaw = D == 256 ? 3 : 4;                        // raw steps
    static constexpr int NB = D / 64;                                    // panels of 64 elements
    static constexpr int kRows = 128 * NT;
    static constexpr int kBlocks = N / kPagedBlock;                      // blocks of 16 tokens of a step
    static constexpr int kUnpackWarps = kBlocks * NB < 8 ? kBlocks * NB : 8;
    static constexpr int kItems = kBlocks * NB / kUnpackWarps;           // (block, panel) pairs of a warp and step
    static constexpr int kPanelQ = 128 * 128, kPanelKV = N * 128;        // bytes
    static constexpr int kQ = NT * NB * kPanelQ, kSlot = NB * kPanelKV, kRawStep = kBlocks * paged_block_bytes(D);
    static constexpr int kMaxSegments = 64;                              // of a CTA between two meetings
    static constexpr int kOffQ = 0, kOffKV = kQ, kOffRaw = kOffKV + kSlots * kSlot, kOffPre = kOffRaw + kRaw * kRawStep;
    static constexpr uint32_t kS = 0, kO = NT * 2 * N;                   // columns of tensor memory: two buffers of S per tile, O
};
constexpr int kTileThreads = 640;
constexpr int kTileOverhead = 6;                                         // a segment without steps, in steps (three ragged prompts of up to 4096: 444 us with 5, 447 with 6, 450 with 7, 455 with 8; a prompt of 4096: 166, 168, 168, 169)

constexpr int kSharedTileSpan = 8;                                       // the least span of the stretches of paged_shared.cuh: a part of a tile is up to 256 rows to write and to join

struct TileSegment {
    int32_t head, row0, n_rows, t0, pos0, end, step0, n, slot;           // rows of the sequence row0 .. (n_rows of it), row 0's token and position, keys [.., end) that one of them sees, steps step0 .. + n
    int64_t table;                                                       // (offset of the sequence's row of the page table)
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes)   // (the rest of the 16: zeros)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float* r)
{
    // the load and its wait form one statement so that no use of r[] can be scheduled between them
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
                 "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]),
                   "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
                   "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31]), "=f"(r[32]), "=f"(r[33]), "=f"(r[34]), "=f"(r[35]),
                   "=f"(r[36]), "=f"(r[37]), "=f"(r[38]), "=f"(r[39]), "=f"(r[40]), "=f"(r[41]), "=f"(r[42]), "=f"(r[43]), "=f"(r[44]), "=f"(r[45]), "=f"(r[46]), "=f"(r[47]),
                   "=f"(r[48]), "=f"(r[49]), "=f"(r[50]), "=f"(r[51]), "=f"(r[52]), "=f"(r[53]), "=f"(r[54]), "=f"(r[55]), "=f"(r[56]), "=f"(r[57]), "=f"(r[58]), "=f"(r[59]),
                   "=f"(r[60]), "=f"(r[61]), "=f"(r[62]), "=f"(r[63])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16_async(uint32_t taddr, const uint32_t r[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// 32 bytes in one store.
__device__ __forceinline__ void store32(void* p, const uint32_t r[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
template <int R> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }
constexpr int kTileRegisters = 96;                                       // of a thread at launch: 5 x 96 = 2 x 128 + 2 x 80 + 64 per four warps
// A wait of a whole warp: its lanes agree on the outcome (what follows is warp-collective).
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t code) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, code)); }

__device__ __forceinline__ int tile_length(int steps) { return steps > 0 ? steps + kTileOverhead : 0; }

// Steps of N keys that the rows [row0, row0 + kRows) of a sequence see: *first the first of them.  rows_all rows of len tokens, n_rows (times group) of them served.
template <int N, int kRows>
__device__ __forceinline__ int tile_steps(int row0, int n_rows, int rows_all, int len, int held, int group, int window, int* first)
{
    const int pos0 = len - rows_all, i0 = row0 / group, i1 = (min(row0 + kRows, n_rows) - 1) / group;
    const int end = min(min(pos0 + i1 + 1, len), held);
    *first = 0;
    if (row0 >= n_rows || end <= 0) return 0;
    if (window > 0) *first = (int)max((int64_t)pos0 + i0 + 1 - window, (int64_t)0) / N;
    return max(0, (int)(((unsigned)end + N - 1) / N) - *first);
}

// Steps of N keys that the rows [row0, row0 + kRows) of a stretch see, *end the keys that they see.
template <int N, int kRows>
__device__ __forceinline__ int stretch_steps(const AttnStretch& v, int row0, int group, int* end)
{
    const int n_rows = v.rows * group;
    *end = 0;
    if (row0 >= n_rows) return 0;
    *end = min(v.pos0 + (min(row0 + kRows, n_rows) - 1) / group + 1, v.end);
    return *end <= 0 ? 0 : max(0, (int)(((unsigned)*end + N - 1) / N) - v.first / N);
}

template <int D, AttnCap CAP, AttnKind KIND = kAttnAll>
__global__ void __launch_bounds__(kTileThreads, 1) paged_tiles_kernel(const PagedAttnParams p)
{
    using T = TileShape<D>;
    constexpr int NT = T::NT, N = T::N, NB = T::NB;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    int* pre = reinterpret_cast<int*>(smem + T::kOffPre);                // [B + 1]: length of the row tiles (per head) before sequence b
    __shared__ __align__(8) uint64_t bars[2 * T::kSlots + 2 * T::kRaw + 15];
    __shared__ TileSegment segs[T::kMaxSegments];
    __shared__ int n_segs;
    __shared__ int64_t round_end;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort_flag[4];
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, c = lane & 3;
    const uint32_t bar0 = smem_u32(bars);
    // barriers: operand slots and raw steps full and empty; S, P and O per buffer (2 t + slot); Q per tile; the end
    constexpr int NS = T::kSlots, NR = T::kRaw;
    const auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    const auto empty = [&](uint32_t s) { return bar0 + 8 * (NS + s); };
    const auto rf = [&](uint32_t s) { return bar0 + 8 * (2 * NS + s); };
    const auto re = [&](uint32_t s) { return bar0 + 8 * (2 * NS + NR + s); };
    const uint32_t bar1 = bar0 + 8 * (2 * NS + 2 * NR);
    const auto sf = [&](int s) { return bar1 + 8 * s; };
    const auto pf = [&](int s) { return bar1 + 8 * (4 + s); };
    const auto of = [&](int s) { return bar1 + 8 * (8 + s); };
    const auto qf = [&](int t) { return bar1 + 8 * (12 + t); };
    const uint32_t done = bar1 + 8 * 14;
    const uint32_t sbase = smem_u32(smem);
    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(full(s), T::kUnpackWarps); mbar_init(empty(s), 1); }
        for (int s = 0; s < NR; ++s) { mbar_init(rf(s), 1); mbar_init(re(s), T::kUnpackWarps); }
        for (int s = 0; s < 4; ++s) { mbar_init(sf(s), 1); mbar_init(pf(s), 4); mbar_init(of(s), 1); }
        mbar_init(qf(0), 4); mbar_init(qf(1), 4);
        mbar_init(done, 2);
        abort_flag[0] = abort_flag[1] = abort_flag[2] = abort_flag[3] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 16) tmem_alloc(smem_u32(&tmem_slot), 512);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) abort_flag[2] = abort_flag[3] = 1;                     // (from here on, waiting counts against the time limit)

    const PagedBatch& bt = p.batch;
    const int held = (int)min((int64_t)bt.table_width << (bt.log2_blocks + 4), (int64_t)INT32_MAX);
    const int n_seqs = KIND == kAttnShared ? p.v1 - p.v0 : bt.B;
    if constexpr (KIND == kAttnShared) {
        for (int v = tid; v <= n_seqs; v += kTileThreads) pre[v] = p.lengths[p.v0 + v] - p.lengths[p.v0];
    } else {
        // ---- the plan: the length of every sequence, their sums
        for (int b = warp; b < bt.B; b += kTileThreads / 32) {
            int t0, first, sum = 0;
            const int rows_all = paged_rows(bt, b, &t0), n_rows = min(rows_all, p.max_q) * p.group, len = bt.kv_len[b];
            for (int r = lane; r * T::kRows < n_rows; r += 32) sum += tile_length(tile_steps<N, T::kRows>(r * T::kRows, n_rows, rows_all, len, held, p.group, p.window, &first));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) pre[b + 1] = sum;
        }
        if (tid == 0) pre[0] = 0;
        __syncthreads();
        if (warp == 0) {
            int carry = 0;
            for (int b0 = 0; b0 < bt.B; b0 += 32) {
                int v = b0 + lane < bt.B ? pre[b0 + lane + 1] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int u = __shfl_up_sync(0xffffffffu, v, o);
                    if (lane >= o) v += u;
                }
                v += carry;
                if (b0 + lane < bt.B) pre[b0 + lane + 1] = v;
                carry = __shfl_sync(0xffffffffu, v, 31);
            }
        }
        // rows of row tiles that see nothing at all: zeros (there are none unless the first or the last row tile is one)
        for (int b = blockIdx.x; b < bt.B; b += gridDim.x) {
            int t0, first;
            const int rows_all = paged_rows(bt, b, &t0), n_rows = min(rows_all, p.max_q) * p.group, len = bt.kv_len[b];
            if (n_rows <= 0) continue;
            const auto steps = [&](int row) { return tile_steps<N, T::kRows>(row / T::kRows * T::kRows, n_rows, rows_all, len, held, p.group, p.window, &first); };
            if (steps(0) > 0 && steps(n_rows - 1) > 0) continue;
            for (int64_t e = tid; e < (int64_t)n_rows * bt.h_kv * (D / 8); e += kTileThreads) {
                const int m = (int)(e % (D / 8)), row = (int)(e / (D / 8) % n_rows), head = (int)(e / (D / 8) / n_rows), i = row / p.group;
                if (steps(row) == 0) *reinterpret_cast<uint4*>(p.out + (int64_t)(t0 + i) * p.out_ld + (int64_t)(head * p.group + row - i * p.group) * D + 8 * m) = make_uint4(0, 0, 0, 0);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);
    const int64_t total = (int64_t)pre[n_seqs] * bt.h_kv, span = max((total + p.grid - 1) / p.grid, (int64_t)(KIND == kAttnShared ? kSharedTileSpan : 1));
    const int64_t w_first = (int64_t)blockIdx.x * span, w_end = min(total, w_first + span);
    if (KIND != kAttnShared && tid == 16 * 32) p.split[blockIdx.x] = make_int4(-1, 0, 0, 0);

    // Rounds of at most kMaxSegments segments; every role has a loop of its own.
    struct Round { int64_t w; uint32_t it0, seg0, steps; int n; bool on; } rd{w_first, 0, 0, 0, 0, w_first < w_end};
    const auto begin_round = [&]() {                                     // (the list is complete)
        __syncwarp();
        __syncthreads();
        rd.n = n_segs;
        rd.steps = 0;
        for (int s = 0; s < rd.n; ++s) rd.steps += segs[s].n;
    };
    const auto end_round = [&]() {
        __syncwarp();
        __syncthreads();
        rd.w = round_end;
        rd.it0 += rd.steps;                                              // steps and segments before the next round
        rd.seg0 += rd.n;
        rd.on = rd.w < w_end && !abort_flag[0];
        __syncthreads();                                                 // (the list may be written again)
    };
    if (warp < 8) {
        more_registers<128>();
        while (rd.on && warp >= 4 * NT) { begin_round(); end_round(); }
        while (rd.on) {
        begin_round();
            // ================================================================ softmax: thread = row
            const int t = NT == 2 ? warp >> 2 : 0, wq = warp & 3, in_tile = 32 * wq + lane;
            const uint32_t lanes = (uint32_t)(32 * wq) << 16, to = tmem + lanes + T::kO + D * t;
            constexpr float kLog2e = 1.4426950408889634f;
            const float mag = fabsf(p.scale), cc = CAP ? 1.f : fmaxf(mag * kLog2e, 1e-30f), margin = kWeightRange / cc;   // weights exp2(cc (x - m)); (cc never 0: hidden scores are -infinity)
            const SoftCap cap(mag, p.softcap);
            // this warp's 32 rows of the tile, copied without waiting, D / 8 lanes' worth of a row side by side; a lane knows where its own row lies
            const auto request_q = [&](const TileSegment& s) {
                constexpr int kChunks = D / 8, kRowsAt = 32 / kChunks, kUnroll = D == 256 ? 4 : 32;   // (whole at d_h <= 128: rolled, the loop below it got 5 % slower)
                const int mine = s.row0 + 128 * t + in_tile, i = mine / p.group;
                const int64_t at = mine < s.n_rows ? (int64_t)(s.t0 + i) * p.q_ld + (int64_t)(s.head * p.group + mine - i * p.group) * D : -1;
                const int sub = lane / kChunks, ch = lane - sub * kChunks;
#pragma unroll kUnroll
                for (int r0 = 0; r0 < 32; r0 += kRowsAt) {
                    const int row = 32 * wq + r0 + sub;
                    const int64_t from = __shfl_sync(0xffffffffu, at, r0 + sub);
                    cp_async16(sbase + T::kOffQ + (t * NB + (ch >> 3)) * T::kPanelQ + row * 128 + (((ch & 7) ^ (row & 7)) << 4), p.q + max(from, (int64_t)0) + 8 * ch, from >= 0 ? 16 : 0);
                }
            };
            const auto hand_q = [&]() {
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(qf(t));
            };
            if (rd.n > 0) { request_q(segs[0]); hand_q(); }
            const bool wide_out = ((reinterpret_cast<uintptr_t>(p.out) | (uintptr_t)(p.out_ld * 2)) & 31) == 0;
            uint32_t it = rd.it0;
            bool ok = true;
            for (int si = 0; si < rd.n && ok; ++si) {
                const TileSegment s = segs[si];
                const int rr = s.row0 + 128 * t + in_tile, i = rr / p.group, pos = s.pos0 + i;
                // (a row behind the sequence's last, whose result nobody looks at, sees all: it does not send its warp through the hiding below)
                const int last = rr < s.n_rows ? min(pos, s.end - 1) : INT32_MAX, lowest = p.window > 0 && rr < s.n_rows ? pos - p.window : -1;
                float m = -1e30f;
                float2 l[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                const int32_t* table = bt.table + s.table;
                const int end_block = (int)(((unsigned)s.end + kPagedBlock - 1) / kPagedBlock);
                const auto page_of = [&](int step) {                     // (lane: the page of the block `lane` from that step on; any page for blocks behind the last: no row sees their tokens, and the table may end there)
                    const int block = step * T::kBlocks + lane;
                    return block < end_block ? table[block >> bt.log2_blocks] : 0;
                };
                constexpr int kAhead = 32 / T::kBlocks;                  // steps of one look-up
                int pg = page_of(s.step0);
                uint32_t held_blocks = 0;
                for (int j = 0; j < s.n; ++j, ++it) {
                    if (j % kAhead == 0) {
                        held_blocks = __ballot_sync(0xffffffffu, pg >= 0 && pg < bt.n_pages);
                        pg = page_of(s.step0 + j + kAhead);
                    }
                    const uint32_t blocks = (held_blocks >> (T::kBlocks * (j % kAhead))) & ((1u << T::kBlocks) - 1);
                    const int slot = 2 * t + (it & 1);
                    if (!warp_wait(sf(slot), (it >> 1) & 1, abort_flag, 0xA00 + slot)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t ts = tmem + lanes + T::kS + N * slot;
                    float x[N];
#pragma unroll
                    for (int e = 0; e < N; e += 64) tmem_ld64(ts + e, x + e);
                    if (CAP) cap.on<CAP, N>(x);
                    const int hi = last - (s.step0 + j) * N, lo = lowest - (s.step0 + j) * N;
                    if (__any_sync(0xffffffffu, hi < N - 1 || lo >= 0) || blocks != (1u << T::kBlocks) - 1) {
                        // one bit per key: up to hi, above lo, of blocks with a page
                        uint64_t see = hi < 0 ? 0 : hi >= 63 ? ~0ull : (2ull << hi) - 1;
                        if (lo >= 0) see &= lo >= 63 ? 0 : ~0ull << (lo + 1);
#pragma unroll
                        for (int k = 0; k < T::kBlocks; ++k)
                            if (!(blocks >> k & 1)) see &= ~(0xffffull << (16 * k));
                        const uint32_t half[2] = {(uint32_t)see, (uint32_t)(see >> 32)};
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (!(half[e >> 5] & 1u << (e & 31))) x[e] = -INFINITY;
                    }
                    float mx[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                    for (int e = 4; e < N; e += 4) {
                        mx[0] = fmaxf(mx[0], x[e]); mx[1] = fmaxf(mx[1], x[e + 1]);
                        mx[2] = fmaxf(mx[2], x[e + 2]); mx[3] = fmaxf(mx[3], x[e + 3]);
                    }
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    if (__any_sync(0xffffffffu, top - m > margin)) {     // m is raised, and with it the scale of the sums
                        const float mn = fmaxf(fmaf(margin, -kWeightLift / kWeightRange, top), m), f = exp2_fast((m - mn) * cc);
                        m = mn;
                        l[0].x *= f; l[0].y *= f; l[1].x *= f; l[1].y *= f;
                        if (j > 0) {
                            // (S of this step is complete before the values of the one before)
                            if (!warp_wait(of(2 * t + ((it - 1) & 1)), ((it - 1) >> 1) & 1, abort_flag, 0xA10 + t)) { ok = false; break; }
                            tc_fence_after();
#pragma unroll 1
                            for (int d = 0; d < D; d += 16) {
                                uint32_t o[16];
                                tmem_ld16(to + d, o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st16_async(to + d, o);
                            }
                        }
                    }
#pragma unroll
                    for (int e = 0; e < N; e += 32) {
                        uint32_t h[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            // (the difference first: x cc - cm with one rounding is not the difference of two scores where cm, a rounded product, is off by powers of two: scores from 2^26 on; 2 % of the time)
                            float2 y = add2(make_float2(x[e + 2 * k], x[e + 2 * k + 1]), make_float2(-m, -m));
                            if (!CAP) y = mul2(y, make_float2(cc, cc));
                            x[e + 2 * k] = y.x;
                            x[e + 2 * k + 1] = y.y;
                        }
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[e + k] = exp2_fast(x[e + k]);
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            l[k & 1] = add2(l[k & 1], make_float2(x[e + 2 * k], x[e + 2 * k + 1]));
                            const __half2 ab = __floats2half2_rn(x[e + 2 * k], x[e + 2 * k + 1]);
                            h[k] = *reinterpret_cast<const uint32_t*>(&ab);
                        }
                        tmem_st16_async(ts + e / 2, h);
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pf(slot));
                }
                if (!ok) break;
                if (si + 1 < rd.n) request_q(segs[si + 1]);              // (every product with this segment's queries is complete)
                const bool landed = warp_wait(of(2 * t + ((it - 1) & 1)), ((it - 1) >> 1) & 1, abort_flag, 0xA20 + t);
                if (si + 1 < rd.n) hand_q();
                if (!landed) { ok = false; break; }
                tc_fence_after();
                const float sum = (l[0].x + l[0].y) + (l[1].x + l[1].y);
                if (KIND == kAttnShared && s.slot < 0) {
                    const int64_t row = attn_row(p, -1 - s.slot, s.t0 + i, s.head, rr - i * p.group);
#pragma unroll 1
                    for (int d = 0; d < D; d += 32) {
                        uint32_t o[32];
                        tmem_ld32(to + d, o);
                        if (rr < s.n_rows)
#pragma unroll
                            for (int e = 0; e < 4; ++e) store32(p.row_o + row * D + d + 8 * e, o + 8 * e);
                    }
                    if (rr < s.n_rows) p.row_ml[row] = make_float2(m * cc, sum);
                } else if (s.slot < 0) {
                    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                    __half* dst = p.out + (int64_t)(s.t0 + i) * p.out_ld + (int64_t)(s.head * p.group + rr - i * p.group) * D;
#pragma unroll 1
                    for (int d = 0; d < D; d += 32) {
                        uint32_t o[32];
                        tmem_ld32(to + d, o);
                        uint32_t h[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const __half2 y = __floats2half2_rn(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
                            h[e] = *reinterpret_cast<const uint32_t*>(&y);
                        }
                        if (rr < s.n_rows) {
#pragma unroll
                            for (int e = 0; e < 4; e += 2) {
                                if (wide_out) store32(dst + d + 8 * e, h + 4 * e);
                                else {
                                    *reinterpret_cast<uint4*>(dst + d + 8 * e) = make_uint4(h[4 * e], h[4 * e + 1], h[4 * e + 2], h[4 * e + 3]);
                                    *reinterpret_cast<uint4*>(dst + d + 8 * e + 8) = make_uint4(h[4 * e + 4], h[4 * e + 5], h[4 * e + 6], h[4 * e + 7]);
                                }
                            }
                        }
                    }
                } else {
                    float* part = p.partial + (int64_t)(2 * blockIdx.x + s.slot) * (T::kRows * (D + 2));
                    const int row = 128 * t + in_tile;
#pragma unroll 1
                    for (int d = 0; d < D; d += 32) {
                        uint32_t o[32];
                        tmem_ld32(to + d, o);
                        if (KIND == kAttnShared && rr >= s.n_rows) continue;   // (nobody reads it)
#pragma unroll
                        for (int e = 0; e < 4; ++e) store32(part + row * D + d + 8 * e, o + 8 * e);
                    }
                    part[T::kRows * D + row] = m * cc;
                    part[T::kRows * D + T::kRows + row] = sum;
                }
                tc_fence_before();
            }
        end_round();
        }
    } else if (warp < 16) {
        fewer_registers<80>();
        while (rd.on && warp >= 8 + T::kUnpackWarps) { begin_round(); end_round(); }
        while (rd.on) {
        begin_round();
            // ================================================================ unpack: K and V of every step from the raw blocks to the operands' layout
            const uint32_t sign = p.scale < 0.f ? 0x80008000u : 0u;
            const int uw = warp - 8;                                     // this warp's (block, panel) pairs: pair kItems * uw + i, panels innermost
            const auto put = [&](uint8_t* row, int chunk, uint32_t word, uint32_t scale) {
                uint32_t h[4];
                unpack_int4_word(word, h);
                *reinterpret_cast<uint4*>(row + chunk * 16) = make_uint4(h2_mul(h[0], scale), h2_mul(h[1], scale), h2_mul(h[2], scale), h2_mul(h[3], scale));
            };
            for (uint32_t q = 0; q < rd.steps; ++q) {
                const uint32_t it = rd.it0 + q, rs = it % NR, nk = 2 * it, nv = 2 * it + 1, sk = nk % NS, sv = nv % NS;
                if (!warp_wait(rf(rs), (it / NR) & 1, abort_flag, 0xA30 + rs)) break;
                uint4 kw[T::kItems], vw[T::kItems];
                uint2 ks[T::kItems], vs[T::kItems];
#pragma unroll
                for (int i = 0; i < T::kItems; ++i) {
                    const int item = T::kItems * uw + i, blk = item / NB, pn = item % NB;
                    const uint8_t* src = smem + T::kOffRaw + rs * T::kRawStep + blk * paged_block_bytes(D);
                    kw[i] = *reinterpret_cast<const uint4*>(src + 512 * pn + 16 * lane);
                    ks[i] = *reinterpret_cast<const uint2*>(src + paged_k_scales(D) + g * (8 * NB) + 8 * pn);
                    ks[i].x ^= sign; ks[i].y ^= sign;                    // (a negative scale of the scores)
                    vw[i] = *reinterpret_cast<const uint4*>(src + paged_v_data(D) + 512 * pn + 16 * lane);
                    vs[i] = *reinterpret_cast<const uint2*>(src + paged_v_scales(D) + (2 * pn + (g >> 2)) * 32 + 8 * c);
                }
                fence_async_smem();                                      // (these reads before the copy that the arrival allows: without it a copy overtook them, now and then)
                __syncwarp();
                if (lane == 0) mbar_arrive(re(rs));
                if (!warp_wait(empty(sk), ((nk / NS) & 1) ^ 1, abort_flag, 0xA40)) break;
#pragma unroll
                for (int i = 0; i < T::kItems; ++i) {
                    const int item = T::kItems * uw + i, blk = item / NB, pn = item % NB;
                    uint8_t* panel = smem + T::kOffKV + sk * T::kSlot + pn * T::kPanelKV + (16 * blk + g) * 128;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {                        // (the group by the row's parity: 8 lanes of a store have 8 chunks)
                        const bool second = (k ^ g) & 1;
                        const uint32_t sc = second ? ks[i].y : ks[i].x;
                        const int chunk = ((second ? 4 : 0) + c) ^ g;
                        put(panel, chunk, second ? kw[i].y : kw[i].x, __byte_perm(sc, sc, 0x1010));
                        put(panel + 8 * 128, chunk, second ? kw[i].w : kw[i].z, __byte_perm(sc, sc, 0x3232));
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(full(sk));
                if (!warp_wait(empty(sv), ((nv / NS) & 1) ^ 1, abort_flag, 0xA41)) break;
#pragma unroll
                for (int i = 0; i < T::kItems; ++i) {
                    const int item = T::kItems * uw + i, blk = item / NB, pn = item % NB;
                    uint8_t* panel = smem + T::kOffKV + sv * T::kSlot + pn * T::kPanelKV;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int row = 2 * c + (k & 1) + 8 * (k >> 1);
                        const uint32_t sc = k & 2 ? vs[i].y : vs[i].x, word = k == 0 ? vw[i].x : k == 1 ? vw[i].y : k == 2 ? vw[i].z : vw[i].w;
                        put(panel + (16 * blk + row) * 128, g ^ (row & 7), word, __byte_perm(sc, sc, k & 1 ? 0x3232 : 0x1010));
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(full(sv));
            }
        end_round();
        }
    } else {
        fewer_registers<64>();                                           // (one instruction for the four warps)
        while (rd.on && warp == 16) {
        // ---- the next segments: (sequence, row tile, KV head), and the part of the steps that lies in the span
        {
            int n = 0;
            int64_t ww = rd.w;
            while (ww < w_end && n < T::kMaxSegments) {
                int lo = 0, hi = n_seqs;                                 // pre[lo] * h_kv <= ww < pre[hi] * h_kv
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if ((int64_t)pre[mid] * bt.h_kv <= ww) lo = mid;
                    else hi = mid;
                }
                int t0, rows_all = 0, n_rows, len = 0, unused;
                AttnStretch v;
                if constexpr (KIND == kAttnShared) {
                    v = p.stretches[p.v0 + lo];
                    t0 = v.t0;
                    n_rows = v.rows * p.group;
                } else {
                    rows_all = paged_rows(bt, lo, &t0);
                    n_rows = min(rows_all, p.max_q) * p.group;
                    len = bt.kv_len[lo];
                }
                int64_t local = ww - (int64_t)pre[lo] * bt.h_kv;
                int r = 0, steps = 0, first = 0;
                for (int r0 = 0;; r0 += 32) {                            // the row tile: sums over 32 at a time
                    int f;
                    const int mine = KIND == kAttnShared ? stretch_steps<N, T::kRows>(v, (r0 + lane) * T::kRows, p.group, &unused)
                                                         : tile_steps<N, T::kRows>((r0 + lane) * T::kRows, n_rows, rows_all, len, held, p.group, p.window, &f);
                    int run = tile_length(mine);
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int u = __shfl_up_sync(0xffffffffu, run, o);
                        if (lane >= o) run += u;
                    }
                    const uint32_t beyond = __ballot_sync(0xffffffffu, (int64_t)run * bt.h_kv > local);
                    if (beyond) {
                        const int at = __ffs(beyond) - 1;
                        r = r0 + at;
                        steps = __shfl_sync(0xffffffffu, mine, at);
                        first = KIND == kAttnShared ? v.first / N : __shfl_sync(0xffffffffu, f, at);
                        local -= (int64_t)(__shfl_sync(0xffffffffu, run, at) - tile_length(steps)) * bt.h_kv;
                        break;
                    }
                    local -= (int64_t)__shfl_sync(0xffffffffu, run, 31) * bt.h_kv;
                }
                const int length = tile_length(steps), head0 = (int)(local / length);
                int ua = (int)(local - (int64_t)head0 * length);
                for (int head = head0; head < bt.h_kv && ww < w_end && n < T::kMaxSegments; ++head, ua = 0) {
                    const int ub = (int)min((int64_t)length, ua + (w_end - ww)), sa = max(ua - kTileOverhead, 0), sb = max(ub - kTileOverhead, 0);
                    if (sb > sa) {
                        const bool whole = sa == 0 && sb == steps;
                        if (KIND == kAttnShared && lane == 0) {
                            int end;
                            stretch_steps<N, T::kRows>(v, r * T::kRows, p.group, &end);
                            segs[n] = TileSegment{head, r * T::kRows, n_rows, t0, v.pos0, end, first + sa, sb - sa, whole ? (p.v0 + lo < p.n_groups ? -1 : -2) : sa > 0 ? 0 : 1, v.seq * bt.table_ld};
                        } else if (lane == 0) {
                            segs[n] = TileSegment{head, r * T::kRows, n_rows, t0, len - rows_all, min(len - rows_all + (min((r + 1) * T::kRows, n_rows) - 1) / p.group + 1, held), first + sa, sb - sa, whole ? -1 : sa > 0 ? 0 : 1, lo * bt.table_ld};
                            if (sa == 0 && !whole) p.split[blockIdx.x] = make_int4(lo, head, r, (int)((ww - ua + length - 1) / span));
                        }
                        ++n;
                    }
                    ww += ub - ua;
                }
            }
            if (lane == 0) round_end = ww;
            if (lane == 0) n_segs = n;
        }
        begin_round();
        {
            // ================================================================ S = Q K^T: the warp runs the loop together, one lane issues
            constexpr uint32_t kIdesc = umma_idesc_f16(N);
            const uint32_t q_lo = umma_desc_lo(sbase + T::kOffQ), k_lo = umma_desc_lo(sbase + T::kOffKV);
            uint32_t it = rd.it0;
            bool ok = true;
            for (int si = 0; si < rd.n && ok; ++si) {
                const int steps = segs[si].n;
                for (int t = 0; t < NT && ok; ++t) ok = warp_wait(qf(t), (rd.seg0 + si) & 1, abort_flag, 0xA50 + t);
                for (int j = 0; j < steps && ok; ++j, ++it) {
                    const uint32_t n = 2 * it, at = n % NS, kd = k_lo + at * (T::kSlot >> 4), sd = tmem + T::kS + N * (it & 1);
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait_hot(full(at), (n / NS) & 1, abort_flag, 0xA60)))) break;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int slot = 2 * t + (it & 1);
                        // (the weights of step it - 2 lay in this buffer)
                        if (it >= 2 && !(ok = __all_sync(0xffffffffu, mbar_wait_hot(of(slot), ((it >> 1) & 1) ^ 1, abort_flag, 0xA64 + slot)))) break;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int pn = 0; pn < NB; ++pn)
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    umma_f16_lo(sd + 2 * N * t, q_lo + (t * NB + pn) * (T::kPanelQ >> 4) + 2 * k, kd + pn * (T::kPanelKV >> 4) + 2 * k, kIdesc, pn + k > 0);
                            umma_commit(sf(slot));
                            if (t == NT - 1) umma_commit(empty(at));
                        }
                        __syncwarp();
                    }
                }
            }
        }
        end_round();
        }
        while (rd.on && warp == 17) {
        begin_round();
        {
            // ================================================================ O += P V
            constexpr uint32_t kIdesc = umma_idesc_f16(D) | (1u << 16);  // (V is transposed)
            const uint32_t v_lo = ((sbase + T::kOffKV) >> 4) | ((uint32_t)(T::kPanelKV >> 4) << 16);
            uint32_t it = rd.it0;
            bool ok = true;
            for (int si = 0; si < rd.n && ok; ++si) {
                const int steps = segs[si].n;
                for (int j = 0; j < steps && ok; ++j, ++it) {
                    const uint32_t n = 2 * it + 1, at = n % NS, vd = v_lo + at * (T::kSlot >> 4), pd = tmem + T::kS + N * (it & 1), add = j > 0;
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait_hot(full(at), (n / NS) & 1, abort_flag, 0xA70)))) break;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int slot = 2 * t + (it & 1);
                        if (!(ok = __all_sync(0xffffffffu, mbar_wait_hot(pf(slot), (it >> 1) & 1, abort_flag, 0xA80 + slot)))) break;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < N / 16; ++k) umma_f16_ta(tmem + T::kO + D * t, pd + 2 * N * t + 8 * k, vd + (2048 >> 4) * k, kIdesc, k > 0 ? 1u : add);
                            umma_commit(of(slot));
                            if (t == NT - 1) umma_commit(empty(at));
                        }
                        __syncwarp();
                    }
                }
            }
        }
        end_round();
        }
        while (rd.on && warp == 18) {
        begin_round();
        {
            // ================================================================ the raw blocks: pages of eight steps looked up at once (lane kBlocks * step + block), eight steps ahead
            constexpr uint32_t kWindow = 32 / T::kBlocks;
            int si = 0, j = 0, si_w = 0, j_w = 0, pages = 0, pages_next = -1;
            const auto look_up = [&]() {
                int sl = si_w, jl = j_w + lane / T::kBlocks;
                while (sl < rd.n && jl >= segs[sl].n) jl -= segs[sl++].n;
                pages_next = -1;
                if (sl < rd.n) {
                    const int block = (segs[sl].step0 + jl) * T::kBlocks + (lane & (T::kBlocks - 1));
                    if (block < (int)(((unsigned)segs[sl].end + kPagedBlock - 1) / kPagedBlock)) pages_next = bt.table[segs[sl].table + (block >> bt.log2_blocks)];
                }
                j_w += kWindow;
                while (si_w < rd.n && j_w >= segs[si_w].n) j_w -= segs[si_w++].n;
            };
            look_up();
            uint32_t q = 0;
            for (; q < rd.steps; ++q) {
                const uint32_t it = rd.it0 + q, rs = it % NR;
                if (q % kWindow == 0) {
                    pages = pages_next >= 0 && pages_next < bt.n_pages ? pages_next : 0;   // (scores of blocks without a page are hidden: any page will do)
                    look_up();
                }
                const int page = __shfl_sync(0xffffffffu, pages, (q % kWindow) * T::kBlocks + (lane & (T::kBlocks - 1))), at = (segs[si].step0 + j) * T::kBlocks + lane;
                const uint8_t* src = bt.pool + ((((int64_t)page * bt.h_kv + segs[si].head) << bt.log2_blocks) + (at & ((1 << bt.log2_blocks) - 1))) * paged_block_bytes(D);
                if (++j == segs[si].n) { j = 0; ++si; }
                if (!warp_wait(re(rs), ((it / NR) & 1) ^ 1, abort_flag, 0xA90 + rs)) break;
                if (lane == 0) mbar_expect_tx(rf(rs), T::kRawStep);
                __syncwarp();
                if (lane < T::kBlocks) bulk_copy_g2s(sbase + T::kOffRaw + rs * T::kRawStep + lane * paged_block_bytes(D), src, paged_block_bytes(D), rf(rs));
            }
            if (abort_flag[0])                                           // (let the copies on their way arrive before the CTA leaves)
                for (uint32_t k = q > NR ? q - NR : 0; k < q; ++k) mbar_wait(rf((rd.it0 + k) % NR), ((rd.it0 + k) / NR) & 1, abort_flag + 1, 0);
        }
        end_round();
        }
        while (rd.on) { begin_round(); end_round(); }                    // (warp 19)
    }
    // every product has to be complete before the memory it reads and writes is given back
    if (warp == 16 || warp == 17) {
        if (elect_one()) umma_commit(done);
        __syncwarp();
        mbar_wait(done, 0, abort_flag + 1, 0);
    }
    __syncthreads();
    if (warp == 16) tmem_dealloc(tmem, 512);
}

}  // namespace ql
