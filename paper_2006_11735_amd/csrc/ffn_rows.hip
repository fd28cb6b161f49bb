// Rows of a stream to 8 bits with a scale each: as they are, or after the residual's addition and the root-mean-square norm.
//   s = x + r (rounded to the stream's type, stored), u = s / sqrt(mean(s^2) + eps) * gamma, scale = max|u| / 127, q = u / scale to nearest, ties to even.
// The root is one factor of the whole row, so it leaves q alone: with v = s * gamma, q = v * (127 / max|v|), and scale = max|v| / 127 / sqrt(...).  One
// reduction brings both the sum of squares and the maximum.
#include "ffn_common.h"

namespace icnn {

// Magnitudes below this are taken for zero as a row's maximum: 127 / max stays finite
constexpr float kLeast = 0x1p-120f;

// Maximum of magnitudes as bit patterns: they are ordered as integers, and a NaN's is above every number's
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// (factor for the numbers, scale of the row).  A row that holds NaN or an infinity, or whose squares do not add up to a finite sum: numbers 0, scale NaN.
__device__ __forceinline__ void row_scale(float squares, uint32_t most, const RowsArgs &a, float *factor, float *scale)
{
    const float m = __builtin_bit_cast(float, most);
    if (most >= 0x7f800000u || !(squares < __builtin_huge_valf())) {
        *factor = 0.f;
        *scale = __builtin_nanf("");
    } else if (m < kLeast) {
        *factor = *scale = 0.f;
    } else {
        *factor = 127.f / m;
        *scale = m / 127.f * (a.gamma ? 1.f / sqrtf(squares / (float)a.c + a.eps) : 1.f);
    }
}

// one number in 8 bits; a factor of 0 makes any number 0
__device__ __forceinline__ int to_byte(float v, float factor)
{
    return factor == 0.f ? 0 : (int)rintf(v * factor);
}

// One workgroup a row, two passes over it.
__global__ __launch_bounds__(256) void rows_kernel(const RowsArgs a)
{
    __shared__ float squares_of[4];
    __shared__ uint32_t most_of[4];
    const long long row = blockIdx.x;
    const int t = threadIdx.x;
    float squares = 0.f;
    uint32_t most = 0;
    for (int i = t; i < a.c; i += 256) {
        float s = load_number(a.x, row * a.ldx + i, a.dtype);
        if (a.res) s = round_number(s + load_number(a.res, row * a.ldr + i, a.dtype), a.dtype);
        if (a.sum) store_number(a.sum, row * a.lds + i, a.dtype, s);
        squares += a.gamma ? s * s : 0.f;
        most = max(most, magnitude(a.gamma ? s * load_number(a.gamma, i, a.gamma_dtype) : s));
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        squares += __shfl_xor(squares, d);
        most = max(most, (uint32_t)__shfl_xor((int)most, d));
    }
    if ((t & 63) == 0) {
        squares_of[t >> 6] = squares;
        most_of[t >> 6] = most;
    }
    __syncthreads();
    squares = (squares_of[0] + squares_of[1]) + (squares_of[2] + squares_of[3]);
    most = max(max(most_of[0], most_of[1]), max(most_of[2], most_of[3]));
    float factor, scale;
    row_scale(squares, most, a, &factor, &scale);
    if (t == 0) a.scale[row] = scale;
    for (int i = t; i < a.c; i += 256) {
        float s;
        if (a.sum) {                                   // (this thread's own, also where it has gone over x or the residual)
            s = load_number(a.sum, row * a.lds + i, a.dtype);
        } else {
            s = load_number(a.x, row * a.ldx + i, a.dtype);
            if (a.res) s = round_number(s + load_number(a.res, row * a.ldr + i, a.dtype), a.dtype);
        }
        if (a.gamma) s *= load_number(a.gamma, i, a.gamma_dtype);
        a.q[row * a.ldq + i] = (int8_t)to_byte(s, factor);
    }
}

hipError_t launch_rows(const RowsArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(rows_kernel, dim3((unsigned)a.rows), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace icnn
