// Angle tables of the rotary embedding: cos and sin of position * frequency for the pairs of a head, times a factor of their own (the scaling of
// long contexts).  The angle is reduced in 64 bits, where it is a number of turns: position * turns per position, less the nearest whole number,
// is exact to 2^-53 of the product, while 32 bits leave a position of 100000 with an angle that is off by 2^-7.
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
    double turns[kRopeTablesMaxPairs];                                   // per position
};

__global__ void __launch_bounds__(256) rope_tables_kernel(const __grid_constant__ RopeTablesParams p)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int quads = p.pairs >> 2;
    const int64_t n = (int64_t)p.n_pos * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int row = (int)(i / quads), j = 4 * (int)(i - (int64_t)row * quads);
        float c[4], s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double t = (double)(p.first + row) * p.turns[j + e];
            sincospif(2.f * (float)(t - rint(t)), s + e, c + e);
        }
        *reinterpret_cast<float4*>(p.cos_t + (int64_t)row * p.pairs + j) = make_float4(c[0] * p.magnitude, c[1] * p.magnitude, c[2] * p.magnitude, c[3] * p.magnitude);
        *reinterpret_cast<float4*>(p.sin_t + (int64_t)row * p.pairs + j) = make_float4(s[0] * p.magnitude, s[1] * p.magnitude, s[2] * p.magnitude, s[3] * p.magnitude);
    }
}

}  // namespace ql
