// What the kernels of products with 4-bit weights share.
#pragma once
#include "ffn_common.h"

namespace icnn {

constexpr int kBlockNumbers = 32, kBlockBytes = 16;

// 16 numbers of a block in 8 bits, times 16 (two's complement in the upper half of each byte): numbers 0 .. 15 are the bytes' lower halves, 16 .. 31 the upper ones
template <bool HIGH>
__device__ __forceinline__ v4i sixteen_of(const v4i &block)
{
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (int)((HIGH ? (unsigned)block[i] : (unsigned)block[i] << 4) & 0xf0f0f0f0u);
    return r;
}

// Scale i: its number as it is, and over 16 (exact, but for numbers that leave float32 downwards) for the sums of sixteen_of's numbers
__device__ __forceinline__ float group_scale(const void *p, long long i, int dtype) { return load_number(p, i, dtype) * 0.0625f; }

__device__ __forceinline__ float scale_of(uint32_t bits, int dtype) { return value_of(bits, dtype) * 0.0625f; }

// Bits of scale i, two bytes or four
template <bool WIDE>
__device__ __forceinline__ uint32_t scale_bits(const void *p, long long i)
{
    return WIDE ? ((const uint32_t *)p)[i] : ((const uint16_t *)p)[i];
}

// Numbers k .. k + 15 of a row of K >= 16 in two steps, so that no load hangs on a condition: sixteen that are there, and of those what k asks for, zeros behind
// the row's end (left: numbers from k on)
__device__ __forceinline__ v4i load_there(const int8_t *row, int k, int K) { return *(const v4i_any *)(row + min(k, K - 16)); }

__device__ __forceinline__ v4i put_right(v4i v, int left)
{
    if (left <= 0) return v4i{};
    if (left >= 16) return v;
    const int by = 16 - left;                              // bytes in front that belong to the piece before
    if (by & 8) v = v4i{v[2], v[3], 0, 0};
    if (by & 4) v = v4i{v[1], v[2], v[3], 0};
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (int)__builtin_amdgcn_alignbyte(i < 3 ? v[i + 1] : 0, v[i], by & 3);
    return r;
}

// Outputs n .. n + 3 of row m from their sums over the groups
template <bool GATED>
__device__ __forceinline__ void finish_four_s4(const LinearS4Args &a, const float (&s)[4], const float (&s2)[4], int m, int n)
{
    const float xs = a.xs[m];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = s[e] * xs + (a.bias ? a.bias[min(n + e, a.N - 1)] : 0.f);
    activate_all(v, a.act, a.dtype);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < a.N) {
            if (GATED) v[e] *= s2[e] * xs + (a.bias2 ? a.bias2[n + e] : 0.f);
            else if (a.res) v[e] += load_number(a.res, m * a.ldr + n + e, a.dtype);
            store_number(a.y, m * a.ldy + n + e, a.dtype, v[e]);
        }
}

hipError_t launch_tokens_s4(const LinearS4Args &a, hipStream_t st);
hipError_t launch_few_s4(const LinearS4Args &a, hipStream_t st);
// (a file for each size of a group: they take long to compile)
hipError_t launch_tiled_s4_32(const LinearS4Args &a, int tile, hipStream_t st);
hipError_t launch_tiled_s4_64(const LinearS4Args &a, int tile, hipStream_t st);
hipError_t launch_tiled_s4_128(const LinearS4Args &a, int tile, hipStream_t st);
hipError_t launch_tiled_s4_256(const LinearS4Args &a, int tile, hipStream_t st);

}  // namespace icnn
