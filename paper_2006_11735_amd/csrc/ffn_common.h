// What the kernels of the feed-forward operators in 8 bits share: their arguments, numbers of the stream's types, activations.
#pragma once
#include "icnn_device.h"

namespace icnn {

constexpr int kF32 = 3, kF16 = 4, kBf16 = 5;      // icnn_dtype of a stream

// Rows to 8 bits with a scale each (see ffn_rows.hip)
struct RowsArgs {
    const void *x, *res, *gamma;    // gamma null: rows as they are, no norm
    void *sum;
    int8_t *q;
    float *scale;
    long long rows, ldx, ldr, lds, ldq;
    int c, dtype, gamma_dtype;
    float eps;
};

// A product of 8-bit rows and 8-bit weights, or the two of a gated layer (see ffn_linear.hip)
struct LinearArgs {
    const int8_t *x, *w, *w2;       // w2 null: one product.  Else y = act(first) * second
    const float *xs, *ws, *ws2, *bias, *bias2;
    const void *res;
    void *y;
    long long ldx, ldw, ldr, ldy;
    int M, N, K;
    int act, dtype;
};

hipError_t launch_rows(const RowsArgs &a, hipStream_t st);
hipError_t launch_linear(const LinearArgs &a, hipStream_t st);
bool few_linear_takes(const LinearArgs &a);
hipError_t launch_few_linear(const LinearArgs &a, hipStream_t st);
bool tiled_linear_takes(const LinearArgs &a);
hipError_t launch_tiled_linear(const LinearArgs &a, hipStream_t st);

typedef int v4i_any __attribute__((ext_vector_type(4), aligned(1)));       // (global memory takes 16 bytes at any address)
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float load_number(const void *p, long long i, int dtype)
{
    if (dtype == kF32) return ((const float *)p)[i];
    if (dtype == kF16) return (float)((const _Float16 *)p)[i];
    return __builtin_bit_cast(float, (uint32_t)((const uint16_t *)p)[i] << 16);
}

// (to nearest, ties to even, as the stream's 16-bit types have it; a NaN stays one)
__device__ __forceinline__ void store_number(void *p, long long i, int dtype, float v)
{
    if (dtype == kF32) ((float *)p)[i] = v;
    else if (dtype == kF16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

__device__ __forceinline__ float round_number(float v, int dtype)
{
    return dtype == kF32 ? v : dtype == kF16 ? (float)(_Float16)v : (float)(__bf16)v;
}

// icnn_act.  The logistic function stands for 1 / (1 + exp(-v)): exp overflows to infinity below v = -88 and its reciprocal is the limit, 0.  The tanh
// form of GELU is v times the logistic function of 2 sqrt(2 / pi) (v + 0.044715 v^3), since (1 + tanh t) / 2 = 1 / (1 + exp(-2 t)).
__device__ __forceinline__ float logistic(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

__device__ __forceinline__ float activate(float v, int act)
{
    if (act == 1) return v < 0.f ? 0.f : v;
    if (act == 2) return v * logistic(v);
    if (act == 3) return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    if (act == 4) return v * logistic(1.5957691216057308f * (v + 0.044715f * v * v * v));
    return v;
}

// 16 numbers k0.. of a row of K, zeros behind its end; reads no byte outside the row
__device__ __forceinline__ v4i load_k16(const int8_t *row, int k0, int K)
{
    if (k0 + 16 <= K) return *(const v4i_any *)(row + k0);
    v4i r = {};
#pragma unroll
    for (int b = 0; b < 16; ++b)
        if (k0 + b < K) r[b >> 2] |= (int)(uint8_t)row[k0 + b] << (8 * (b & 3));
    return r;
}

// One output: y[m][n] from the sums of one product, or two
template <bool GATED>
__device__ __forceinline__ float finish(const LinearArgs &a, int acc, int acc2, float xs, int n)
{
    float v = (float)acc * xs * a.ws[n];
    if (a.bias) v += a.bias[n];
    v = activate(v, a.act);
    if (GATED) {
        float v2 = (float)acc2 * xs * a.ws2[n];
        if (a.bias2) v2 += a.bias2[n];
        v *= v2;
    }
    return v;
}

// Sixteen numbers from p[i] on, in the stream's type
__device__ __forceinline__ void load_sixteen(const void *p, long long i, int dtype, float (&v)[16])
{
    if (dtype == kF32) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const v4f t = *(const v4f_any *)((const float *)p + i + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = t[e];
        }
        return;
    }
    const v4i lo = *(const v4i_any *)((const uint16_t *)p + i), hi = *(const v4i_any *)((const uint16_t *)p + i + 8);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint16_t b = (uint16_t)((uint32_t)(e < 8 ? lo : hi)[(e & 7) >> 1] >> (16 * (e & 1)));
        v[e] = dtype == kF16 ? (float)__builtin_bit_cast(_Float16, b) : __builtin_bit_cast(float, (uint32_t)b << 16);
    }
}

__device__ __forceinline__ void store_sixteen(void *p, long long i, int dtype, const float (&v)[16])
{
    if (dtype == kF32) {
#pragma unroll
        for (int q = 0; q < 4; ++q) *(v4f_any *)((float *)p + i + 4 * q) = v4f{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        return;
    }
    v4i t[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[2 * e], y = v[2 * e + 1];
        const uint32_t b = dtype == kF16 ? __builtin_bit_cast(uint16_t, (_Float16)x) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)y) << 16
                                         : __builtin_bit_cast(uint16_t, (__bf16)x) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y) << 16;
        t[e >> 2][e & 3] = (int)b;
    }
    *(v4i_any *)((uint16_t *)p + i) = t[0];
    *(v4i_any *)((uint16_t *)p + i + 8) = t[1];
}

// Sixteen scales or biases from p[n] on, the last one again behind the row's end
__device__ __forceinline__ void load_column(const float *p, int n, int N, float (&v)[16])
{
    if (n + 16 <= N) {
        load_sixteen(p, n, kF32, v);
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = p[min(n + e, N - 1)];
    }
}

__device__ __forceinline__ void scale_sixteen(const int (&c)[16], float xs, const float *ws, const float *bias, int n, int N, float (&v)[16])
{
    float t[16];
    load_column(ws, n, N, t);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = (float)c[e] * xs * t[e];
    if (bias) {
        load_column(bias, n, N, t);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] += t[e];
    }
}

// Outputs n .. n + 15 of row m (both inside) from their sums c, gated also c2: everything behind the sums, y written
template <bool GATED>
__device__ __forceinline__ void finish_sixteen(const LinearArgs &a, const int (&c)[16], const int (&c2)[16], int m, int n)
{
    float v[16], u[16];
    const float xs = a.xs[m];
    scale_sixteen(c, xs, a.ws, a.bias, n, a.N, v);
    if (a.act != 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = activate(v[e], a.act);
    }
    if (GATED) {
        scale_sixteen(c2, xs, a.ws2, a.bias2, n, a.N, u);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] *= u[e];
    }
    const long long at = m * a.ldy + n, res_at = m * a.ldr + n;
    if (n + 16 <= a.N) {
        if (!GATED && a.res) {
            load_sixteen(a.res, res_at, a.dtype, u);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] += u[e];
        }
        store_sixteen(a.y, at, a.dtype, v);
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (n + e < a.N) {
                if (!GATED && a.res) v[e] += load_number(a.res, res_at + e, a.dtype);
                store_number(a.y, at + e, a.dtype, v[e]);
            }
    }
}

}  // namespace icnn
