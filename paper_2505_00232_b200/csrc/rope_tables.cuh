// Angle tables of the rotary embedding: cos and sin of position * frequency for the pairs of a head, times a factor of their own (the scaling of
// long contexts).
//
// The angle is a number of turns in 64-bit fixed point: position * (turns per position * 2^64), of which only the fraction of a turn matters, so
// the product may overflow; its upper half, 32 bits of a turn, is what two integer multiplications give (32-bit floating point would leave position 100000
// with an angle that is off by 2^-7).  Its quarter turn chooses sine or cosine and the signs; the rest, at most an eighth of a turn either way, goes through
// the Taylor polynomials of degree 9 and 8, whose next terms are below 2.6e-8 there.  Bound: HBM (8 bytes written per pair and position).  A thread keeps its 4 pairs and goes
// over the positions, so that their frequencies are read once.  131072 positions of 64 pairs: 34 us with sincospif on a 64-bit reduction, 12 so.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace ql {

constexpr int kRopeTablesMaxPairs = 256;
struct RopeTablesParams {
    float* cos_t;
    float* sin_t;                // [n_pos, pairs]
    int32_t first, n_pos, pairs; // pairs: a multiple of 8
    float magnitude;
    uint64_t turns[kRopeTablesMaxPairs];                                 // per position, in 2^-64
};

__global__ void __launch_bounds__(256) rope_tables_kernel(const __grid_constant__ RopeTablesParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int quads = p.pairs >> 2, per_block = 256 / quads, sub = threadIdx.x / quads, j = 4 * (threadIdx.x - sub * quads);
    if (sub >= per_block) return;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) { hi[e] = (uint32_t)(p.turns[j + e] >> 32); lo[e] = (uint32_t)p.turns[j + e]; }
    for (int64_t row = (int64_t)blockIdx.x * per_block + sub; row < p.n_pos; row += (int64_t)gridDim.x * per_block) {
        const uint32_t pos = (uint32_t)(p.first + row);
        float c[4], s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t turn = pos * hi[e] + __umulhi(pos, lo[e]);    // 2^-32 of a turn
            const uint32_t quarter = (turn + 0x20000000u) >> 30;
            const float x = (float)(int32_t)(turn - (quarter << 30)) * 1.4629180792671596e-9f, z = x * x;   // 2 pi / 2^32
            const float sn = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
            const float cs = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320))));
            const float a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;                              // a quarter turn on: sin -> cos, cos -> -sin
            s[e] = (quarter & 2 ? -a : a) * p.magnitude;
            c[e] = ((quarter + 1) & 2 ? -b : b) * p.magnitude;
        }
        *reinterpret_cast<float4*>(p.cos_t + row * p.pairs + j) = make_float4(c[0], c[1], c[2], c[3]);
        *reinterpret_cast<float4*>(p.sin_t + row * p.pairs + j) = make_float4(s[0], s[1], s[2], s[3]);
    }
}

}  // namespace ql
