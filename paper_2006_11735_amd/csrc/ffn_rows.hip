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

// Eight numbers of the stream from p[i] on, to and from float32
template <int DT>
__device__ __forceinline__ void stream_eight(const void *p, long long i, float (&v)[8])
{
    if (DT == kF32) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const v4f t = __builtin_nontemporal_load((const v4f_any *)((const float *)p + i + 4 * q));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = t[e];
        }
        return;
    }
    const v4i t = __builtin_nontemporal_load((const v4i_any *)((const uint16_t *)p + i));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint16_t b = (uint16_t)((uint32_t)t[e >> 1] >> (16 * (e & 1)));
        v[e] = DT == kF16 ? (float)__builtin_bit_cast(_Float16, b) : __builtin_bit_cast(float, (uint32_t)b << 16);
    }
}

// (rounds v as it stores it)
template <int DT>
__device__ __forceinline__ v4i pack_eight(float (&v)[8])
{
    v4i t;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint16_t b[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float &x = v[2 * e + h];
            b[h] = DT == kF16 ? __builtin_bit_cast(uint16_t, (_Float16)x) : __builtin_bit_cast(uint16_t, (__bf16)x);
            x = DT == kF16 ? (float)__builtin_bit_cast(_Float16, b[h]) : __builtin_bit_cast(float, (uint32_t)b[h] << 16);
        }
        t[e] = (int)(b[0] | (uint32_t)b[1] << 16);
    }
    return t;
}

typedef int v2i_any __attribute__((ext_vector_type(2), aligned(1)));

// Rows that fit a workgroup's registers: read once.  T threads a row (a wave, with neither LDS nor a barrier, or all 256), V times eight numbers a thread.
template <int DT, int T, int V>
__global__ __launch_bounds__(256) void rows_held_kernel(const RowsArgs a)
{
    const long long row = (long long)blockIdx.x * (256 / T) + threadIdx.x / T;
    const int t = threadIdx.x % T;
    if (T == 64 && row >= a.rows) return;
    float v[V][8], squares = 0.f;
    uint32_t most = 0;
    // all loads first
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int i = 8 * (k * T + t);
        if (i + 8 <= a.c) {
            stream_eight<DT>(a.x, row * a.ldx + i, v[k]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = i + e < a.c ? load_number(a.x, row * a.ldx + i + e, DT) : 0.f;
        }
    }
    if (a.res) {
        float u[V][8];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int i = 8 * (k * T + t);
            if (i + 8 <= a.c) {
                stream_eight<DT>(a.res, row * a.ldr + i, u[k]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) u[k][e] = i + e < a.c ? load_number(a.res, row * a.ldr + i + e, DT) : 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = round_number(v[k][e] + u[k][e], DT);
    }
    if (a.sum) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int i = 8 * (k * T + t);
            if (i + 8 <= a.c) {
                if (DT == kF32) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        *(v4f_any *)((float *)a.sum + row * a.lds + i + 4 * q) = v4f{v[k][4 * q], v[k][4 * q + 1], v[k][4 * q + 2], v[k][4 * q + 3]};
                } else {
                    *(v4i_any *)((uint16_t *)a.sum + row * a.lds + i) = pack_eight<DT>(v[k]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (i + e < a.c) store_number(a.sum, row * a.lds + i + e, DT, v[k][e]);
            }
        }
    }
    if (a.gamma) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int i = 8 * (k * T + t);
            float gm[8];
            if (i + 8 <= a.c) {
                if (DT == kF32 || a.gamma_dtype == DT) stream_eight<DT>(a.gamma, i, gm);
                else stream_eight<kF32>(a.gamma, i, gm);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) gm[e] = i + e < a.c ? load_number(a.gamma, i + e, a.gamma_dtype) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                squares += v[k][e] * v[k][e];
                v[k][e] *= gm[e];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[k][e]));
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        squares += __shfl_xor(squares, d);
        most = max(most, (uint32_t)__shfl_xor((int)most, d));
    }
    if (T == 256) {
        __shared__ float squares_of[4];
        __shared__ uint32_t most_of[4];
        if ((t & 63) == 0) {
            squares_of[t >> 6] = squares;
            most_of[t >> 6] = most;
        }
        __syncthreads();
        squares = (squares_of[0] + squares_of[1]) + (squares_of[2] + squares_of[3]);
        most = max(max(most_of[0], most_of[1]), max(most_of[2], most_of[3]));
    }
    float factor, scale;
    row_scale(squares, most, a, &factor, &scale);
    if (t == 0) a.scale[row] = scale;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int i = 8 * (k * T + t);
        uint32_t b[2] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e >> 2] |= (uint32_t)(to_byte(v[k][e], factor) & 255) << (8 * (e & 3));
        if (i + 8 <= a.c) {
            *(v2i_any *)(a.q + row * a.ldq + i) = v2i_any{(int)b[0], (int)b[1]};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e < a.c) a.q[row * a.ldq + i + e] = (int8_t)(b[e >> 2] >> (8 * (e & 3)));
        }
    }
}

template <int DT>
static void launch_rows_of(const RowsArgs &a, hipStream_t st)
{
    const dim3 waves((unsigned)((a.rows + 3) / 4)), groups((unsigned)a.rows), block(256);
    if (a.c <= 512) hipLaunchKernelGGL((rows_held_kernel<DT, 64, 1>), waves, block, 0, st, a);
    else if (a.c <= 1024) hipLaunchKernelGGL((rows_held_kernel<DT, 64, 2>), waves, block, 0, st, a);
    else if (a.c <= 2048) hipLaunchKernelGGL((rows_held_kernel<DT, 256, 1>), groups, block, 0, st, a);
    else if (a.c <= 4096) hipLaunchKernelGGL((rows_held_kernel<DT, 256, 2>), groups, block, 0, st, a);
    else if (a.c <= 8192) hipLaunchKernelGGL((rows_held_kernel<DT, 256, 4>), groups, block, 0, st, a);
    else if (a.c <= 16384) hipLaunchKernelGGL((rows_held_kernel<DT, 256, 8>), groups, block, 0, st, a);
    else hipLaunchKernelGGL(rows_kernel, groups, block, 0, st, a);
}

hipError_t launch_rows(const RowsArgs &a, hipStream_t st)
{
    if (a.dtype == kF32) launch_rows_of<kF32>(a, st);
    else if (a.dtype == kF16) launch_rows_of<kF16>(a, st);
    else launch_rows_of<kBf16>(a, st);
    return hipGetLastError();
}

}  // namespace icnn
