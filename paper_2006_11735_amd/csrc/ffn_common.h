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

}  // namespace icnn
