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

// Which sequence row t of the call belongs to, and its position there; false for a row of none.  Every thread of the CTA takes part.
__device__ __forceinline__ bool paged_locate(const PagedBatch& p, int t, int* seq, int* position)
{
    __shared__ int found[2];
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    for (int b = threadIdx.x; b < p.B; b += blockDim.x) {
        int first;
        const int n = paged_rows(p, b, &first);
        if (t >= first && t - first < n) {
            found[0] = b;
            found[1] = p.kv_len[b] - n + (t - first);
        }
    }
    __syncthreads();
    *seq = found[0];
    *position = found[1];
    return found[0] >= 0;
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
__device__ __forceinline__ uint32_t paged_quantise(const uint4& u, __half* scale)
{
    float f[8];
    paged_unpack8(u, f);
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(f[i]));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const float s = fminf(__half2float(__float2half_rn(__fdiv_rn(amax, 7.f))), 9352.f);
    *scale = __float2half_rn(s);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int q = s > 0.f ? __float2int_rn(fminf(fmaxf(__fdiv_rn(f[i], s), -7.f), 7.f)) : 0;   // (clamped, then rounded: the same, 7 is a whole number)
        w |= (uint32_t)(q + 8) << (4 * ((i >> 1) + 4 * (i & 1)));
    }
    return w;
}

// One CTA per row of the call (and, for few rows, per piece of its heads); d / 8 lanes per head, 8 elements each: one 16-byte load, the partner of the
// two-halves layout by a shuffle, the group's maximum by two.  Every product and sum of the rotation is one rounded fp32 operation, the result is
// rounded to fp16 (what the calls that it stands for write), and that is quantised: the integers do not depend on the compiler's contractions.
__global__ void __launch_bounds__(kPagedThreads) paged_append_kernel(const PagedAppendParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t = blockIdx.x, d = p.d;
    int b, pos;
    if (!paged_locate(p.batch, t, &b, &pos) || pos < 0) return;
    const int log2_lanes = 31 - __clz(d >> 3), lane = threadIdx.x & 31, m = lane & ((1 << log2_lanes) - 1);
    const int h_kv = p.batch.h_kv, rows = p.h_q + 2 * h_kv, per_pass = kPagedThreads >> log2_lanes;
    const int half = p.rot >> 1, hl = half >> 3;                         // the lanes of the first half's elements
    const int64_t at = (int64_t)min(pos, p.n_pos - 1) * half;
    const int block_bytes = paged_block_bytes(d);

    for (int base = blockIdx.y * per_pass; base < rows; base += gridDim.y * per_pass) {
        const int r = base + (threadIdx.x >> log2_lanes);
        const int kind = r < p.h_q ? 0 : r < p.h_q + h_kv ? 1 : 2, head = kind == 0 ? r : kind == 1 ? r - p.h_q : r - p.h_q - h_kv;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            const __half* src = kind == 0 ? p.q + t * p.q_ld : kind == 1 ? p.k + t * p.k_ld : p.v + t * p.v_ld;
            u = *reinterpret_cast<const uint4*>(src + (int64_t)head * d + 8 * m);
        }
        if (p.cos_t) {
            float x[8], y[8], o[8];
            paged_unpack8(u, x);
            if (p.interleaved) {
                if (kind < 2 && 8 * m < p.rot) {
                    const float4 c = __ldg(reinterpret_cast<const float4*>(p.cos_t + at + 4 * m)), s = __ldg(reinterpret_cast<const float4*>(p.sin_t + at + 4 * m));
                    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        o[2 * i] = __fsub_rn(__fmul_rn(x[2 * i], cc[i]), __fmul_rn(x[2 * i + 1], ss[i]));
                        o[2 * i + 1] = __fadd_rn(__fmul_rn(x[2 * i + 1], cc[i]), __fmul_rn(x[2 * i], ss[i]));
                    }
                }
            } else {
                const int partner = lane - m + (m < hl ? m + hl : m < 2 * hl ? m - hl : m);
                uint4 w;
                w.x = __shfl_sync(0xffffffffu, u.x, partner);
                w.y = __shfl_sync(0xffffffffu, u.y, partner);
                w.z = __shfl_sync(0xffffffffu, u.z, partner);
                w.w = __shfl_sync(0xffffffffu, u.w, partner);
                paged_unpack8(w, y);
                if (kind < 2 && 8 * m < p.rot) {
                    const bool low = m < hl;
                    const int i0 = 8 * (low ? m : m - hl);
                    float c[8], s[8];
#pragma unroll
                    for (int i = 0; i < 8; i += 4) {
                        *reinterpret_cast<float4*>(c + i) = __ldg(reinterpret_cast<const float4*>(p.cos_t + at + i0 + i));
                        *reinterpret_cast<float4*>(s + i) = __ldg(reinterpret_cast<const float4*>(p.sin_t + at + i0 + i));
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = __fadd_rn(__fmul_rn(x[i], c[i]), __fmul_rn(low ? -y[i] : y[i], s[i]));
                }
            }
            if (kind < 2 && 8 * m < p.rot) {
                __half2* h = reinterpret_cast<__half2*>(&u);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(o[2 * i], o[2 * i + 1]);
            }
        }
        __half scale;
        const uint32_t word = paged_quantise(u, &scale);                 // (every lane: it shuffles)
        if (r >= rows) continue;
        if (kind == 0) {
            *reinterpret_cast<uint4*>(p.q_out + t * p.q_out_ld + (int64_t)head * d + 8 * m) = u;
        } else if (uint8_t* block = paged_block(p.batch, b, pos, head, block_bytes)) {
            const int tt = pos & 15;
            *reinterpret_cast<uint32_t*>(block + (kind == 1 ? paged_k_word(m, tt) : paged_v_word(m, tt, d))) = word;
            if ((m & 3) == 0) *reinterpret_cast<__half*>(block + (kind == 1 ? paged_k_scale(m, tt, d) : paged_v_scale(m, tt, d))) = scale;
        }
    }
}

struct PagedReadParams {
    PagedBatch batch;
    __half* k;                   // [T, h_kv, d]
    __half* v;
    int32_t d;
};

// fp16(q * s) of the tokens of a call, zeros where the table gives them no page: one CTA per row, 8 elements per lane.
__global__ void __launch_bounds__(kPagedThreads) paged_read_kernel(const PagedReadParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t = blockIdx.x, d = p.d;
    int b, pos;
    if (!paged_locate(p.batch, t, &b, &pos)) return;
    const int lanes = d >> 3, n = p.batch.h_kv * lanes;
    for (int i = threadIdx.x; i < 2 * n; i += kPagedThreads) {
        const bool value = i >= n;
        const int r = value ? i - n : i, head = r / lanes, m = r - head * lanes, tt = pos & 15;
        const uint8_t* block = paged_block(p.batch, b, pos, head, paged_block_bytes(d));
        uint4 u = make_uint4(0, 0, 0, 0);
        if (block) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(block + (value ? paged_v_word(m, tt, d) : paged_k_word(m, tt)));
            const float s = __half2float(*reinterpret_cast<const __half*>(block + (value ? paged_v_scale(m, tt, d) : paged_k_scale(m, tt, d))));
            __half2* h = reinterpret_cast<__half2*>(&u);
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = __floats2half2_rn((float)((int)((w >> (4 * e)) & 15) - 8) * s, (float)((int)((w >> (4 * e + 16)) & 15) - 8) * s);
        }
        *reinterpret_cast<uint4*>((value ? p.v : p.k) + ((int64_t)t * p.batch.h_kv + head) * d + 8 * m) = u;
    }
}

}  // namespace ql
