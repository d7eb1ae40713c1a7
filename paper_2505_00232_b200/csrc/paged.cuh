// A paged KV cache held in 4 bits: its layout, the kernel that appends tokens (with the rotation of queries and keys on the way) and the one
// that reads positions back.
//
// 32 consecutive elements of a head's key or value vector share a scale, one per TOKEN and group, as in the int4 weights of this library:
//     s = min(fp16(amax / 7), 9352),   q = clamp(round-half-even(v / s), -7, 7)           (IEEE fp32 operations)
// (a group whose scale rounds to zero holds zeros; 9352 is the largest fp16 number whose sevenfold is finite in fp16, so that q * s always is).
//
// A page holds page_size tokens (a power of two from 16 on) of every KV head; [page][head][page_size / 16] blocks of 16 tokens, each 1152 bytes
// per 64 elements of the head:
//     K integers   per 64 elements 32 lanes x 16 bytes: lane 4 (t % 8) + c holds the elements 8 c .. 8 c + 7 of both groups, of the tokens t and
//                  t + 8: the operand of m16n8k16 with tokens as rows, after the unpack
//     K scales     [t % 8][group][t / 8] fp16
//     V integers   per 64 elements 32 lanes x 16 bytes: lane 4 g + c holds the elements 8 g .. 8 g + 7 of the tokens 2c, 2c + 1, 2c + 8, 2c + 9:
//                  the operand with elements as rows (two words give two tokens for each of 8 elements)
//     V scales     [group][c][2c, 2c + 1, 2c + 8, 2c + 9] fp16
// A word holds 8 elements of ONE token (so that tokens are written without reading): element i in nibble i / 2 + 4 (i % 2), as q + 8; the masks of
// the unpack then give neighbours in order.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace ql {

constexpr int kPagedBlock = 16;                                          // tokens of a block
__host__ __device__ constexpr int paged_block_bytes(int d) { return 1152 * (d >> 6); }
__host__ __device__ constexpr int paged_k_scales(int d) { return 512 * (d >> 6); }       // offsets in a block
__host__ __device__ constexpr int paged_v_data(int d) { return 576 * (d >> 6); }
__host__ __device__ constexpr int paged_v_scales(int d) { return 1088 * (d >> 6); }

// Byte offsets in a block of the word that holds elements 8 m .. 8 m + 7 of token t (0 to 15), and of the scale of their group.
__host__ __device__ __forceinline__ int paged_k_word(int m, int t) { return (m >> 3) * 512 + ((t & 7) * 4 + (m & 3)) * 16 + ((t >> 3) * 2 + ((m & 7) >> 2)) * 4; }
__host__ __device__ __forceinline__ int paged_k_scale(int m, int t, int d) { return paged_k_scales(d) + ((t & 7) * (d >> 5) + (m >> 2)) * 4 + (t >> 3) * 2; }
__host__ __device__ __forceinline__ int paged_v_word(int m, int t, int d) { return paged_v_data(d) + (m >> 3) * 512 + ((m & 7) * 4 + ((t & 7) >> 1)) * 16 + ((t & 1) + 2 * (t >> 3)) * 4; }
__host__ __device__ __forceinline__ int paged_v_scale(int m, int t, int d) { return paged_v_scales(d) + ((m >> 2) * 4 + ((t & 7) >> 1)) * 8 + ((t & 1) + 2 * (t >> 3)) * 2; }

// The batch of a call: sequence b has the rows q_start[b] .. q_start[b + 1] - 1 of the call, its last tokens, and kv_len[b] tokens with them; token
// j of it lies in page table[b * table_ld + j / page_size].
struct PagedBatch {
    uint8_t* pool;
    const int32_t* table;
    const int32_t* kv_len;
    const int32_t* q_start;
    int32_t B, T, table_width, n_pages, log2_blocks, h_kv;               // T: rows of the call; 2^log2_blocks blocks of 16 tokens in a page
    int64_t table_ld;
};

// The rows of sequence b that a call serves; 0 where q_start does not name rows of the call.
__device__ __forceinline__ int paged_rows(const PagedBatch& p, int b, int* first)
{
    const int s = p.q_start[b], e = p.q_start[b + 1];
    *first = s;
    return s < 0 || e > p.T || e < s ? 0 : e - s;
}
// The block that holds token j of sequence b for a head; null where the table does not give it a page of the pool.
__device__ __forceinline__ uint8_t* paged_block(const PagedBatch& p, int b, int j, int head, int block_bytes)
{
    const int block = j >> 4, at = block >> p.log2_blocks;
    if (j < 0 || at >= p.table_width) return nullptr;
    const int page = p.table[b * p.table_ld + at];
    if (page < 0 || page >= p.n_pages) return nullptr;
    return p.pool + ((((int64_t)page * p.h_kv + head) << p.log2_blocks) + (block & ((1 << p.log2_blocks) - 1))) * block_bytes;
}

constexpr int kPagedThreads = 256;
constexpr int kPagedMostRows = 8;                                        // rows of the call that a CTA takes

// Which sequences the rows t0 .. t0 + n - 1 (n <= kPagedMostRows) of the call belong to (seq[i], -1: none), and their positions there.  Every thread of the CTA takes part.
__device__ __forceinline__ void paged_locate(const PagedBatch& p, int t0, int n, int* seq, int* position)
{
    if (threadIdx.x < n) seq[threadIdx.x] = -1;
    __syncthreads();
    for (int b = threadIdx.x; b < p.B; b += blockDim.x) {
        int first;
        const int rows = paged_rows(p, b, &first);
        for (int t = max(first, t0); t < min(first + rows, t0 + n); ++t) {
            seq[t - t0] = b;
            position[t - t0] = (int)max((int64_t)p.kv_len[b] - rows + (t - first), (int64_t)-1);   // (negative: before the first token)
        }
    }
    __syncthreads();
}

struct PagedAppendParams {
    PagedBatch batch;
    const __half* q;             // may be null
    const __half* k;
    const __half* v;
    __half* q_out;
    const float* cos_t;          // [n_pos, rot / 2]; null: no rotation
    const float* sin_t;
    int64_t q_ld, k_ld, v_ld, q_out_ld;
    int32_t h_q, d, n_pos, rot, interleaved;
};

__device__ __forceinline__ void paged_unpack8(const uint4& u, float f[8])
{
    const __half2* h = reinterpret_cast<const __half2*>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = __half22float2(h[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
}

// 8 elements of a group that 4 neighbouring lanes hold: the word, and the group's scale.
// The integers are those of round-half-even of the IEEE quotient, without dividing: for fp16 numbers x and s, x / s below 16 is a tie (a whole number and a half) or at
// least 2^-14 away from one (2 x and an odd multiple of s are multiples of a unit that is at least 2^-12 of the larger), so x r + 384 with the reciprocal r, off by less than
// 2^-18 before it is rounded, once, to a multiple of 2^-15, has the ties exact again.  The scale: fp16(amax * (1 / 7)) is fp16(amax / 7) for every fp16 number.
__device__ __forceinline__ uint32_t paged_quantise(const uint4& u, __half* scale)
{
    const __half2* h2 = reinterpret_cast<const __half2*>(&u);
    const __half2 top = __hmax2(__hmax2(__habs2(h2[0]), __habs2(h2[1])), __hmax2(__habs2(h2[2]), __habs2(h2[3])));
    float amax = fmaxf(__low2float(top), __high2float(top));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const float s = fminf(__half2float(__float2half_rn(__fmul_rn(amax, 1.f / 7))), 9352.f);
    *scale = __float2half_rn(s);
    const float r = s > 0.f ? __frcp_rn(s) : 0.f;
    float f[8];
    paged_unpack8(u, f);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)                                          // the bits of 1.5 * 2^23 and the integer + 8 as the low ones
        b[i] = __float_as_uint(__fadd_rn(fminf(fmaxf(__fmaf_rn(f[i], r, 384.f), 377.f), 391.f), 12582536.f));
    uint32_t w = b[7];                                                   // nibble 7 first; what the upper bits add up to is taken off at the end
    w = w * 16 + b[5]; w = w * 16 + b[3]; w = w * 16 + b[1];
    w = w * 16 + b[6]; w = w * 16 + b[4]; w = w * 16 + b[2]; w = w * 16 + b[0];
    return w - 0x3f400000u;
}

// ROWS rows of the call per CTA, one after the other (and, for few rows, a CTA per piece of the heads); d / 8 lanes per head, 8 elements each: one 16-byte load, the partner of
// the two-halves layout by a shuffle, the group's maximum by two.  A thread has the same elements of several heads: it requests up to kHeads of them at once
// and reads the angles, the same for all heads, once per row.  Every product and sum of the rotation is one rounded fp32 operation, the result is
// rounded to fp16 (what the calls that it stands for write), and that is quantised: the integers do not depend on the compiler's contractions.
// Bound: HBM.
template <int ROWS>
__global__ void __launch_bounds__(kPagedThreads, ROWS > 1 ? 4 : 1) paged_append_kernel(const PagedAppendParams p)
{
    constexpr int kHeads = 3;
    __shared__ int seq[kPagedMostRows], position[kPagedMostRows];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int d = p.d, n = min(ROWS, p.batch.T - (int)blockIdx.x * ROWS);
    paged_locate(p.batch, blockIdx.x * ROWS, n, seq, position);
    const int log2_lanes = 31 - __clz(d >> 3), lane = threadIdx.x & 31, m = lane & ((1 << log2_lanes) - 1);
    const int h_kv = p.batch.h_kv, rows = p.h_q + 2 * h_kv, per_pass = kPagedThreads >> log2_lanes;
    const int half = p.rot >> 1, hl = half >> 3;                         // the lanes of the first half's elements
    const int block_bytes = paged_block_bytes(d);
    const bool turned = p.cos_t && 8 * m < p.rot, low = m < hl;
    const int partner = p.interleaved ? lane : lane - m + (low ? m + hl : m < 2 * hl ? m - hl : m);
    const int angle = p.interleaved ? 4 * m : 8 * (low ? m : m - hl);

    for (int i = 0; i < n; ++i) {
        const int b = seq[i], pos = position[i];
        if (b < 0 || pos < 0) continue;
        const int64_t t = (int64_t)blockIdx.x * ROWS + i;
        float c[8], sn[8];
        if (turned) {
            const int64_t at = (int64_t)min(pos, p.n_pos - 1) * half + angle;
            *reinterpret_cast<float4*>(c) = __ldg(reinterpret_cast<const float4*>(p.cos_t + at));
            *reinterpret_cast<float4*>(sn) = __ldg(reinterpret_cast<const float4*>(p.sin_t + at));
            if (!p.interleaved) {
                *reinterpret_cast<float4*>(c + 4) = __ldg(reinterpret_cast<const float4*>(p.cos_t + at + 4));
                *reinterpret_cast<float4*>(sn + 4) = __ldg(reinterpret_cast<const float4*>(p.sin_t + at + 4));
            }
        }
        const __half *q_row = p.q + t * p.q_ld + 8 * m, *k_row = p.k + t * p.k_ld + 8 * m, *v_row = p.v + t * p.v_ld + 8 * m;
        __half* q_to = p.q_out + t * p.q_out_ld + 8 * m;
        uint8_t* blocks = paged_block(p.batch, b, pos, 0, block_bytes);  // of head 0; the others' lie a head of the page further each
        for (int base = blockIdx.y * per_pass; base < rows; base += gridDim.y * per_pass * kHeads) {
            uint4 u[kHeads];
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
                const int r = base + k * gridDim.y * per_pass + (threadIdx.x >> log2_lanes);
                const __half* src = r < p.h_q ? q_row : r < p.h_q + h_kv ? k_row : v_row;
                const int head = r < p.h_q ? r : r < p.h_q + h_kv ? r - p.h_q : r - p.h_q - h_kv;
                u[k] = r < rows ? *reinterpret_cast<const uint4*>(src + head * d) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
                const int r0 = base + k * gridDim.y * per_pass + (int)((threadIdx.x & ~31u) >> log2_lanes), r = r0 + (lane >> log2_lanes);   // r0: the warp's first head
                if (r0 >= rows) break;
                const bool is_value = r >= p.h_q + h_kv;
                if (p.cos_t && r0 < p.h_q + h_kv) {
                    uint4 w;
                    w.x = __shfl_sync(0xffffffffu, u[k].x, partner);
                    w.y = __shfl_sync(0xffffffffu, u[k].y, partner);
                    w.z = __shfl_sync(0xffffffffu, u[k].z, partner);
                    w.w = __shfl_sync(0xffffffffu, u[k].w, partner);
                    if (turned && !is_value) {
                        float x[8], o[8];
                        paged_unpack8(u[k], x);
                        if (p.interleaved) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                o[2 * e] = __fsub_rn(__fmul_rn(x[2 * e], c[e]), __fmul_rn(x[2 * e + 1], sn[e]));
                                o[2 * e + 1] = __fadd_rn(__fmul_rn(x[2 * e + 1], c[e]), __fmul_rn(x[2 * e], sn[e]));
                            }
                        } else {
                            float y[8];
                            paged_unpack8(w, y);
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] = __fadd_rn(__fmul_rn(x[e], c[e]), __fmul_rn(low ? -y[e] : y[e], sn[e]));
                        }
                        __half2* h = reinterpret_cast<__half2*>(&u[k]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) h[e] = __floats2half2_rn(o[2 * e], o[2 * e + 1]);
                    }
                }
                if (r < p.h_q) *reinterpret_cast<uint4*>(q_to + r * d) = u[k];
                if (!blocks || r0 + (31 >> log2_lanes) < p.h_q) continue;   // (a warp of queries only)
                __half scale;
                const uint32_t word = paged_quantise(u[k], &scale);      // (every lane: it shuffles)
                if (r >= p.h_q && r < rows) {
                    const int head = is_value ? r - p.h_q - h_kv : r - p.h_q, tt = pos & 15;
                    uint8_t* block = blocks + ((int64_t)head << p.batch.log2_blocks) * block_bytes;
                    *reinterpret_cast<uint32_t*>(block + (is_value ? paged_v_word(m, tt, d) : paged_k_word(m, tt))) = word;
                    if ((m & 3) == 0) *reinterpret_cast<__half*>(block + (is_value ? paged_v_scale(m, tt, d) : paged_k_scale(m, tt, d))) = scale;
                }
            }
        }
    }
}

struct PagedReadParams {
    PagedBatch batch;
    __half* k;                   // [T, h_kv, d]
    __half* v;
    int32_t d;
};

__device__ __forceinline__ uint4 paged_values(uint32_t w, __half scale)
{
    uint4 u;
    __half2* h = reinterpret_cast<__half2*>(&u);
    const float s = __half2float(scale);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __floats2half2_rn((float)((int)((w >> (4 * e)) & 15) - 8) * s, (float)((int)((w >> (4 * e + 16)) & 15) - 8) * s);
    return u;
}

// fp16(q * s) of the tokens of a call, zeros where the table gives them no page: ROWS rows per CTA, 8 elements of the key and of the value per lane.
template <int ROWS>
__global__ void __launch_bounds__(kPagedThreads) paged_read_kernel(const PagedReadParams p)
{
    __shared__ int seq[kPagedMostRows], position[kPagedMostRows];
    __shared__ const uint8_t* first_head[kPagedMostRows];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int d = p.d, n = min(ROWS, p.batch.T - (int)blockIdx.x * ROWS), bytes = paged_block_bytes(d);
    paged_locate(p.batch, blockIdx.x * ROWS, n, seq, position);
    if (threadIdx.x < n && seq[threadIdx.x] >= 0) first_head[threadIdx.x] = paged_block(p.batch, seq[threadIdx.x], position[threadIdx.x], 0, bytes);
    __syncthreads();
    const int lanes = d >> 3, per = p.batch.h_kv * lanes;
#pragma unroll 2
    for (int i = threadIdx.x; i < n * per; i += kPagedThreads) {
        const int row = i / per, r = i - row * per, head = r / lanes, m = r - head * lanes;
        if (seq[row] < 0) continue;
        const int tt = position[row] & 15;
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        if (const uint8_t* block = first_head[row]) {
            block += ((int64_t)head << p.batch.log2_blocks) * bytes;
            const uint32_t kw = *reinterpret_cast<const uint32_t*>(block + paged_k_word(m, tt)), vw = *reinterpret_cast<const uint32_t*>(block + paged_v_word(m, tt, d));
            const __half ks = *reinterpret_cast<const __half*>(block + paged_k_scale(m, tt, d)), vs = *reinterpret_cast<const __half*>(block + paged_v_scale(m, tt, d));
            k = paged_values(kw, ks);
            v = paged_values(vw, vs);
        }
        const int64_t to = (((int64_t)blockIdx.x * ROWS + row) * p.batch.h_kv + head) * d + 8 * m;
        *reinterpret_cast<uint4*>(p.k + to) = k;
        *reinterpret_cast<uint4*>(p.v + to) = v;
    }
}

}  // namespace ql
