// Adjusts the logits of an LM head before sampling: penalties for tokens that a row has seen, biases for listed tokens, and a mask of allowed ones.
//
//   x = l;   token seen in the row's history (prompt or output):  x = x > 0 ? x / repetition : x * repetition
//            token seen n > 0 times in the output:                x = x - frequency n - presence
//            token in the row's bias list:                        x = x + bias (the last entry of a token counts)
//            token's mask bit 0:                                  x = -infinity
//
// in fp32, each operation rounded, one rounding to the logits' type.  Bound: HBM (each logit read and written once); few rows: the chain of latencies
// (start of the list -> tokens -> counts -> store).  A CTA owns a tile of a row's vocabulary: it requests its logits, counts the history's tokens
// that fall into the tile in shared memory (integer atomics: the order does not matter), and marks them in a bitmap, so that the pass over the
// logits looks at the counts of marked tokens only.  No table of counts per row is kept or read: the history itself is shorter than the row.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace ql {

constexpr int kLogitsThreads = 256;

struct LogitsParams {
    const void* x;
    void* y;
    int64_t ld, out_ld, mask_ld;
    const int32_t* tokens;       // may be null: no history
    const int32_t* start;        // [rows + 1]
    const int32_t* n_prompt;     // [rows]: this many of a row's tokens are its prompt; null: none
    const float* repetition;     // [rows], null: 1
    const float* presence;       // [rows], null: 0
    const float* frequency;
    const int32_t* bias_ids;     // may be null
    const float* bias_values;
    const int32_t* bias_start;   // [rows + 1]
    const uint32_t* mask;        // may be null: all allowed
    int32_t rows, vocab, n_tokens, n_biases;
};

// TILE tokens of a row's vocabulary per CTA.  T: __half or float, 16 bytes of them at a time (V).
template <typename T, int TILE>
__global__ void __launch_bounds__(kLogitsThreads) adjust_logits_kernel(const LogitsParams p)
{
    constexpr int V = 16 / sizeof(T), kVecs = TILE / (V * kLogitsThreads);
    static_assert(kVecs * V * kLogitsThreads == TILE, "whole vectors");
    extern __shared__ __align__(128) uint8_t smem[];
    uint32_t* count = reinterpret_cast<uint32_t*>(smem);                 // bit 0: in the prompt, above: times in the output
    uint32_t* listed = count + TILE;                                     // number of the token's last bias entry, from 1 (only with biases)
    __shared__ uint32_t marked[TILE / 32 + 1], allowed[TILE / 32 + 1];
    const int tid = threadIdx.x, row = blockIdx.y, t0 = blockIdx.x * TILE, n = min(TILE, p.vocab - t0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // the first `head` tokens of a tile lie before a 16-byte boundary; with input and output aligned alike the rest goes 16 bytes at a time
    const T* x = static_cast<const T*>(p.x) + row * p.ld + t0;
    T* y = static_cast<T*>(p.y) + row * p.out_ld + t0;
    const int off = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == (reinterpret_cast<uintptr_t>(y) & 15);
    const int head = wide ? min(n, (V - off) & (V - 1)) : n, n_vec = (n - head) / V, tail = head + n_vec * V;
    uint4 v[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
        if (tid + k * kLogitsThreads < n_vec) v[k] = *reinterpret_cast<const uint4*>(x + head + (tid + k * kLogitsThreads) * V);

    const uint4 zero = make_uint4(0, 0, 0, 0);
    if (p.tokens)
        for (int i = tid; i < TILE / 4; i += kLogitsThreads) reinterpret_cast<uint4*>(count)[i] = zero;
    if (p.bias_ids)
        for (int i = tid; i < TILE / 4; i += kLogitsThreads) reinterpret_cast<uint4*>(listed)[i] = zero;
    for (int i = tid; i <= TILE / 32; i += kLogitsThreads) {
        marked[i] = 0;
        allowed[i] = p.mask && 32 * i < n ? p.mask[row * p.mask_ld + (t0 >> 5) + i] : 0xffffffffu;
    }
    __syncthreads();
    int b0 = 0;
    if (p.tokens) {
        const int first = max(p.start[row], 0), end = min(p.start[row + 1], p.n_tokens);
        const int prompt_end = p.n_prompt ? (int)min((int64_t)first + max(p.n_prompt[row], 0), (int64_t)p.n_tokens) : first;
#pragma unroll 4
        for (int i = first + tid; i < end; i += kLogitsThreads) {
            const int t = p.tokens[i] - t0;
            if (t >= 0 && t < n) {
                if (i < prompt_end) atomicOr(&count[t], 1u);
                else atomicAdd(&count[t], 2u);
                atomicOr(&marked[t >> 5], 1u << (t & 31));
            }
        }
    }
    if (p.bias_ids) {
        b0 = max(p.bias_start[row], 0);
        const int b1 = min(p.bias_start[row + 1], p.n_biases);
        for (int i = b0 + tid; i < b1; i += kLogitsThreads) {
            const int t = p.bias_ids[i] - t0;
            if (t >= 0 && t < n) {
                atomicMax(&listed[t], (uint32_t)(i - b0 + 1));
                atomicOr(&marked[t >> 5], 1u << (t & 31));
            }
        }
    }
    const float rep = p.repetition ? p.repetition[row] : 1.f, pres = p.presence ? p.presence[row] : 0.f, freq = p.frequency ? p.frequency[row] : 0.f;
    __syncthreads();

    auto adjusted = [&](float l, int t) {                                // a marked token
        const uint32_t c = p.tokens ? count[t] : 0u;
        if (c) l = l > 0.f ? __fdiv_rn(l, rep) : __fmul_rn(l, rep);
        if (c > 1) l = __fsub_rn(__fsub_rn(l, __fmul_rn(freq, (float)(c >> 1))), pres);
        const uint32_t e = p.bias_ids ? listed[t] : 0u;
        if (e) l = __fadd_rn(l, p.bias_values[b0 + (int)e - 1]);
        return l;
    };
    auto single = [&](int t) {
        float l = (float)x[t];
        if (marked[t >> 5] >> (t & 31) & 1) l = adjusted(l, t);
        y[t] = (allowed[t >> 5] >> (t & 31) & 1) ? (T)l : (T)(-INFINITY);
    };
    for (int t = tid; t < head; t += kLogitsThreads) single(t);
    for (int t = tail + tid; t < n; t += kLogitsThreads) single(t);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int i = tid + k * kLogitsThreads, t = head + i * V;
        if (i >= n_vec) break;
        constexpr uint32_t kAll = (1u << V) - 1;
        const uint32_t mark = __funnelshift_r(marked[t >> 5], marked[(t >> 5) + 1], t & 31) & kAll, allow = __funnelshift_r(allowed[t >> 5], allowed[(t >> 5) + 1], t & 31) & kAll;
        T* e = reinterpret_cast<T*>(&v[k]);
        if (mark) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (mark >> j & 1) e[j] = (T)adjusted((float)e[j], t + j);
        }
        if (allow != kAll) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (!(allow >> j & 1)) e[j] = (T)(-INFINITY);
        }
        *reinterpret_cast<uint4*>(y + t) = v[k];
    }
}

}  // namespace ql
