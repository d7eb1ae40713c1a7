// Adjusts the logits of an LM head before sampling: penalties for tokens that a row has seen, biases for listed tokens, and a mask of allowed ones.
//
//   x = l;   token seen in the row's history (prompt or output):  x = x > 0 ? x / repetition : x * repetition
//            token seen n > 0 times in the output:                x = x - frequency n - presence
//            token in the row's bias list:                        x = x + bias (the last entry of a token counts)
//            token's mask bit 0:                                  x = -infinity
//
// in fp32, each operation rounded, one rounding to the logits' type.  Bound: HBM (each logit read and written once); few rows: the chain of latencies
// (start of the list -> tokens -> counts -> store).  No table of counts per row is kept or read: the history itself is shorter than the row.
//
// Few rows (adjust_logits_kernel): a CTA owns a tile of a row's vocabulary.  It requests the tile's logits; goes through the row's history and biases and, for the tokens in the tile,
// counts in shared memory (integer atomics: the order does not matter), marks them in a bitmap and lists every one once; adjusts the listed ones, spread evenly over the
// threads, into shared memory; and passes over the tile with the mask, 16 bytes at a time, taking marked tokens from there.
//
// Many rows: every tile of a row going through its whole history costs more than the logits (256 rows of 128256, histories of 512 to 4096: 65 us with tiles of 8192).  So mask_logits_kernel copies the logits
// under the mask, nothing else (and is left out where there is no mask and nothing to copy), and adjust_seen_kernel, a CTA per row, goes through the history twice: once for a bitmap of what it
// holds, whose bits, counted up to each word, number the distinct tokens; once to count into a table of that many entries; and then adjusts those logits only (the same: 38 us, of 21 for the bytes).
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
    bool masked;                 // mask_logits_kernel comes before adjust_seen_kernel
};

template <typename T> struct LogitBits { using type = uint16_t; };
template <> struct LogitBits<float> { using type = uint32_t; };

// A pair of 16-bit (or one 32-bit) logits whose bit(s) in `allow` are 0 become minus infinity.  V = 8: bits 2 k and 2 k + 1 become masks of 16 bits by the byte
// permutation's replication of a sign; `spread` = allow | allow << 7 holds them 8 bits apart.
template <int V>
__device__ __forceinline__ uint32_t masked_logits(uint32_t x, uint32_t allow, uint32_t spread, int k)
{
    if (V == 4) return allow >> k & 1 ? x : 0xff800000u;
    uint32_t m, r;
    asm("prmt.b32 %0, %1, %1, 0x9988;" : "=r"(m) : "r"(2 * k < 7 ? spread << (7 - 2 * k) : spread));
    asm("lop3.b32 %0, %1, %2, %3, 0xca;" : "=r"(r) : "r"(m), "r"(x), "r"(0xfc00fc00u));   // m ? x : -infinity, bit by bit
    return r;
}

// TILE tokens of a row's vocabulary per CTA.  T: __half or float, 16 bytes of them at a time (V).
template <typename T, int TILE>
__global__ void __launch_bounds__(kLogitsThreads) adjust_logits_kernel(const LogitsParams p)
{
    constexpr int V = 16 / sizeof(T), kVecs = TILE / (V * kLogitsThreads) > 0 ? TILE / (V * kLogitsThreads) : 1, kWords = TILE / 32;
    extern __shared__ __align__(128) uint8_t smem[];
    uint32_t* count = reinterpret_cast<uint32_t*>(smem);                 // [TILE] bit 0: in the prompt, above: times in the output; then the adjusted logit
    uint32_t* listed = count + TILE;                                     // [TILE / 2] 16 bits a token: number of its last bias entry, from 1
    uint16_t* todo = reinterpret_cast<uint16_t*>(listed + TILE / 2);     // [TILE] the marked tokens
    __shared__ uint32_t marked[kWords + 1], allowed[kWords + 1];
    __shared__ int n_todo;
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

    int first = 0, end = 0, prompt_end = 0, b0 = 0, b1 = 0;
    float rep = 1.f, pres = 0.f, freq = 0.f;
    if (p.tokens) {
        first = max(p.start[row], 0);
        end = min(p.start[row + 1], p.n_tokens);
        prompt_end = p.n_prompt ? (int)min((int64_t)first + max(p.n_prompt[row], 0), (int64_t)p.n_tokens) : first;
        if (p.repetition) rep = p.repetition[row];
        if (p.presence) pres = p.presence[row];
        if (p.frequency) freq = p.frequency[row];
    }
    if (p.bias_ids) {
        b1 = min(p.bias_start[row + 1], p.n_biases);
        b0 = max(max(p.bias_start[row], 0), b1 - 65535);                 // (16 bits number the entries)
    }
    const uint4 zero = make_uint4(0, 0, 0, 0);
    if (p.tokens || p.bias_ids)
        for (int i = tid; i < TILE / 4; i += kLogitsThreads) reinterpret_cast<uint4*>(count)[i] = zero;
    if (p.bias_ids)
        for (int i = tid; i < TILE / 8; i += kLogitsThreads) reinterpret_cast<uint4*>(listed)[i] = zero;
    for (int i = tid; i <= kWords; i += kLogitsThreads) {
        marked[i] = 0;
        allowed[i] = p.mask && 32 * i < n ? p.mask[row * p.mask_ld + (t0 >> 5) + i] : 0xffffffffu;
    }
    if (tid == 0) n_todo = 0;
    __syncthreads();
    const auto mark = [&](int t) {
        if (!(atomicOr(&marked[t >> 5], 1u << (t & 31)) >> (t & 31) & 1)) todo[atomicAdd(&n_todo, 1)] = (uint16_t)t;
    };
#pragma unroll 4
    for (int i = first + tid; i < end; i += kLogitsThreads) {
        const int t = p.tokens[i] - t0;
        if (t >= 0 && t < n) {
            if (i < prompt_end) atomicOr(&count[t], 1u);
            else atomicAdd(&count[t], 2u);
            mark(t);
        }
    }
    for (int i = b0 + tid; i < b1; i += kLogitsThreads) {
        const int t = p.bias_ids[i] - t0;
        if (t >= 0 && t < n) {
            const uint32_t mine = (uint32_t)(i - b0 + 1), sh = 16 * (t & 1);
            uint32_t seen = listed[t >> 1];                              // (the largest number stays, whatever the order)
            while ((seen >> sh & 0xffff) < mine) {
                const uint32_t was = atomicCAS(&listed[t >> 1], seen, (seen & ~(0xffffu << sh)) | mine << sh);
                if (was == seen) break;
                seen = was;
            }
            mark(t);
        }
    }
    __syncthreads();
    for (int i = tid; i < n_todo; i += kLogitsThreads) {
        const int t = todo[i];
        const uint32_t c = count[t];
        float l = (float)x[t];
        if (c) l = l > 0.f ? __fdiv_rn(l, rep) : __fmul_rn(l, rep);
        if (c > 1) l = __fsub_rn(__fsub_rn(l, __fmul_rn(freq, (float)(c >> 1))), pres);
        const uint32_t e = p.bias_ids ? listed[t >> 1] >> (16 * (t & 1)) & 0xffff : 0u;
        if (e) l = __fadd_rn(l, p.bias_values[b0 + (int)e - 1]);
        const T r = (T)l;
        count[t] = sizeof(T) == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(&r) : *reinterpret_cast<const uint32_t*>(&r);
    }
    __syncthreads();

    const auto single = [&](int t) {
        T l = x[t];
        if (marked[t >> 5] >> (t & 31) & 1) *reinterpret_cast<typename LogitBits<T>::type*>(&l) = (typename LogitBits<T>::type)count[t];
        y[t] = (allowed[t >> 5] >> (t & 31) & 1) ? l : (T)(-INFINITY);
    };
    for (int t = tid; t < head; t += kLogitsThreads) single(t);
    for (int t = tail + tid; t < n; t += kLogitsThreads) single(t);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int i = tid + k * kLogitsThreads, t = head + i * V;
        if (i >= n_vec) break;
        constexpr uint32_t kAll = (1u << V) - 1;
        const uint32_t mark = __funnelshift_r(marked[t >> 5], marked[(t >> 5) + 1], t & 31) & kAll, allow = __funnelshift_r(allowed[t >> 5], allowed[(t >> 5) + 1], t & 31) & kAll;
        for (uint32_t m = mark; m; m &= m - 1) {
            const int j = __ffs(m) - 1;
            const uint32_t r = count[t + j];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t& u = (&v[k].x)[w];
                if (V == 4) { if (j == w) u = r; }
                else if (j >> 1 == w) u = j & 1 ? __byte_perm(u, r, 0x5410) : __byte_perm(u, r, 0x3254);
            }
        }
        if (p.mask) {
            const uint32_t spread = allow | allow << 7;
#pragma unroll
            for (int w = 0; w < 4; ++w) (&v[k].x)[w] = masked_logits<V>((&v[k].x)[w], allow, spread, w);
        }
        *reinterpret_cast<uint4*>(y + t) = v[k];
    }
}

// y = mask ? x : -infinity, a piece of a row per CTA.
template <typename T>
__global__ void __launch_bounds__(kLogitsThreads) mask_logits_kernel(const LogitsParams p)
{
    constexpr int V = 16 / sizeof(T), kVecs = 4, kPiece = V * kVecs * kLogitsThreads;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, row = blockIdx.y, t0 = blockIdx.x * kPiece, n = min(kPiece, p.vocab - t0);
    const T* x = static_cast<const T*>(p.x) + row * p.ld + t0;
    T* y = static_cast<T*>(p.y) + row * p.out_ld + t0;
    const uint32_t* mask = p.mask ? p.mask + row * p.mask_ld + (t0 >> 5) : nullptr;
    const int words = (n + 31) >> 5, off = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == (reinterpret_cast<uintptr_t>(y) & 15);
    const int head = wide ? min(n, (V - off) & (V - 1)) : n, n_vec = (n - head) / V, tail = head + n_vec * V;
    uint4 v[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
        if (tid + k * kLogitsThreads < n_vec) v[k] = *reinterpret_cast<const uint4*>(x + head + (tid + k * kLogitsThreads) * V);
    const auto single = [&](int t) { y[t] = !mask || (mask[t >> 5] >> (t & 31) & 1) ? x[t] : (T)(-INFINITY); };
    for (int t = tid; t < head; t += kLogitsThreads) single(t);
    for (int t = tail + tid; t < n; t += kLogitsThreads) single(t);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int i = tid + k * kLogitsThreads, t = head + i * V;
        if (i >= n_vec) break;
        if (mask) {
            const uint32_t allow = __funnelshift_r(mask[t >> 5], mask[min((t >> 5) + 1, words - 1)], t & 31) & ((1u << V) - 1), spread = allow | allow << 7;
#pragma unroll
            for (int w = 0; w < 4; ++w) (&v[k].x)[w] = masked_logits<V>((&v[k].x)[w], allow, spread, w);
        }
        *reinterpret_cast<uint4*>(y + t) = v[k];
    }
}

constexpr int kSeenThreads = 512, kSeenTokens = 1 << 17, kSeenWords = kSeenTokens / 32, kSeenEntries = 4096;   // tokens of the vocabulary per CTA; entries of the table
constexpr int kSeenBytes = kSeenWords * 8 + kSeenEntries * 12;
// The tokens of a row's history and biases in a piece of the vocabulary.  Everything up to the first table is done before the kernel before this one (mask_logits_kernel, which passed its own
// wait: what came before it is complete) has to be.
template <typename T>
__global__ void __launch_bounds__(kSeenThreads) adjust_seen_kernel(const LogitsParams p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem);                  // [kSeenWords] tokens that are there
    uint32_t* before = bits + kSeenWords;                                // [kSeenWords] how many of them lie in the words before
    uint32_t* count = before + kSeenWords;                               // [kSeenEntries] bit 0: in the prompt, above: times in the output
    uint32_t* listed = count + kSeenEntries;                             // number of the last bias entry, from 1
    uint32_t* token_of = listed + kSeenEntries;
    __shared__ uint32_t warp_sum[kSeenThreads / 32];
    if (!p.masked) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, row = blockIdx.y, t0 = blockIdx.x * kSeenTokens, n = min(kSeenTokens, p.vocab - t0);
    int first = 0, end = 0, prompt_end = 0, b0 = 0, b1 = 0;
    float rep = 1.f, pres = 0.f, freq = 0.f;
    if (p.tokens) {
        first = max(p.start[row], 0);
        end = min(p.start[row + 1], p.n_tokens);
        prompt_end = p.n_prompt ? (int)min((int64_t)first + max(p.n_prompt[row], 0), (int64_t)p.n_tokens) : first;
        if (p.repetition) rep = p.repetition[row];
        if (p.presence) pres = p.presence[row];
        if (p.frequency) freq = p.frequency[row];
    }
    if (p.bias_ids) {
        b1 = min(p.bias_start[row + 1], p.n_biases);
        b0 = max(max(p.bias_start[row], 0), b1 - 65535);                 // (as for few rows)
    }
    for (int i = tid; i < kSeenWords / 4; i += kSeenThreads) reinterpret_cast<uint4*>(bits)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    // f(number of the entry, token less t0) for the entries in this piece
    const auto each = [&](const int32_t* ids, int from, int to, auto f) {
#pragma unroll 4
        for (int i = from + tid; i < to; i += kSeenThreads) {
            const int token = ids[i];
            const uint32_t t = (uint32_t)token - (uint32_t)t0;
            if (token >= 0 && t < (uint32_t)n) f(i, (int)t);
        }
    };
    const auto set = [&](int, int t) {
        if (!(bits[t >> 5] >> (t & 31) & 1)) atomicOr(&bits[t >> 5], 1u << (t & 31));   // (frequent tokens meet here: looked at first)
    };
    each(p.tokens, first, end, set);
    each(p.bias_ids, b0, b1, set);
    __syncthreads();
    constexpr int kEach = kSeenWords / kSeenThreads;
    uint32_t sum = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) sum += __popc(bits[tid * kEach + k]);
    uint32_t run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, run, o);
        if ((tid & 31) >= o) run += u;
    }
    if ((tid & 31) == 31) warp_sum[tid >> 5] = run;
    __syncthreads();
    run -= sum;
    uint32_t distinct = 0;
    for (int w = 0; w < kSeenThreads / 32; ++w) {
        if (w < tid >> 5) run += warp_sum[w];
        distinct += warp_sum[w];
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        before[tid * kEach + k] = run;
        run += __popc(bits[tid * kEach + k]);
    }
    bool waited = !p.masked;
    const T* x = static_cast<const T*>(p.x) + row * p.ld + t0;
    T* y = static_cast<T*>(p.y) + row * p.out_ld + t0;
    const uint32_t* mask = p.mask ? p.mask + row * p.mask_ld + (t0 >> 5) : nullptr;
    for (uint32_t e0 = 0; e0 < distinct; e0 += kSeenEntries) {           // (a table at a time)
        const uint32_t entries = min(distinct - e0, (uint32_t)kSeenEntries);
        for (uint32_t i = tid; i < entries; i += kSeenThreads) count[i] = listed[i] = 0;
        __syncthreads();
        const auto entry_of = [&](int t) { return before[t >> 5] + __popc(bits[t >> 5] & ((1u << (t & 31)) - 1)) - e0; };
        each(p.tokens, first, end, [&](int i, int t) {
            const uint32_t e = entry_of(t);
            if (e >= entries) return;
            if (i < prompt_end) { if (!(count[e] & 1)) atomicOr(&count[e], 1u); }
            else atomicAdd(&count[e], 2u);
            token_of[e] = t;
        });
        each(p.bias_ids, b0, b1, [&](int i, int t) {
            const uint32_t e = entry_of(t);
            if (e >= entries) return;
            atomicMax(&listed[e], (uint32_t)(i - b0 + 1));
            token_of[e] = t;
        });
        if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
        waited = true;
        __syncthreads();
        for (uint32_t i = tid; i < entries; i += kSeenThreads) {
            const int t = token_of[i];
            const uint32_t c = count[i], e = listed[i];
            if (mask && !(mask[t >> 5] >> (t & 31) & 1)) continue;       // (minus infinity already)
            float l = (float)x[t];
            if (c) l = l > 0.f ? __fdiv_rn(l, rep) : __fmul_rn(l, rep);
            if (c > 1) l = __fsub_rn(__fsub_rn(l, __fmul_rn(freq, (float)(c >> 1))), pres);
            if (e) l = __fadd_rn(l, p.bias_values[b0 + (int)e - 1]);
            y[t] = (T)l;
        }
        __syncthreads();
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
}

}  // namespace ql
