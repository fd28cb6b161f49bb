// What the kernels of the feed-forward operators in 8 bits share: their arguments, numbers of the stream's types, activations.
#pragma once
#include "icnn_device.h"
#include "ffn_plan.h"

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

hipError_t launch_rows(const RowsArgs &a, hipStream_t st);
hipError_t launch_linear(const LinearArgs &a, hipStream_t st);
// kernels of ffn_tokens.hip, ffn_few.hip and ffn_tiled.hip
hipError_t launch_tokens_linear(const LinearArgs &a, hipStream_t st);
hipError_t launch_few_linear(const LinearArgs &a, hipStream_t st);
hipError_t launch_tiled_linear(const LinearArgs &a, const TilePlan &plan, hipStream_t st);

inline LinearTuning linear_tuning() { return {g_tuning.ff_kernel, g_tuning.ff_split}; }

typedef int v4i_any __attribute__((ext_vector_type(4), aligned(1)));       // (global memory takes 16 bytes at any address)
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float load_number(const void *p, long long i, int dtype)
{
    if (dtype == kF32) return ((const float *)p)[i];
    if (dtype == kF16) return (float)((const _Float16 *)p)[i];
    return __builtin_bit_cast(float, (uint32_t)((const uint16_t *)p)[i] << 16);
}

// The same in two steps, so that no branch waits for the load: the bits, and their value
__device__ __forceinline__ uint32_t load_bits(const void *p, long long i, int dtype)
{
    return dtype == kF32 ? ((const uint32_t *)p)[i] : ((const uint16_t *)p)[i];
}

__device__ __forceinline__ float value_of(uint32_t bits, int dtype)
{
    const float f16 = (float)__builtin_bit_cast(_Float16, (uint16_t)bits), other = __builtin_bit_cast(float, dtype == kF32 ? bits : bits << 16);
    return dtype == kF16 ? f16 : other;
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
// The erf form is v times the normal distribution's function F.
// For results in 16 bits by formula 7.1.26 of Abramowitz and Stegun's handbook for 1 - erf(x), x = |v| / sqrt 2 (error below 1.5e-7): 1 - erf(x) =
// (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + p x).
// For float32 results, of which that is off by up to 7e-7 between -1 and 0, by two fits.  Up to |v| = 1.25: F = 1/2 + v P(v^2), where the half leaves nothing of P's
// rounding in sight.  Beyond: F(-|v|) = exp(-v^2 / 2) R(t), t = 1 / (1 + 0.4 |v|), with a relative error that holds to where F leaves float32.  P (degree 5, off F by
// 1e-8 of it) and R (degree 7 without a constant, 4.6e-8) are least-maximum fits to F in 64 bits.
// (24 x 2048 -> 8192 in float32 8.1 us, by the other formula 7.65; 300 x 1000 -> 1300 8.4 and 7.65; in 16 bits, which do not show the difference, as before.)
__device__ __forceinline__ float logistic(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

constexpr int kGeluF32 = 5;        // (beside the numbers of icnn_act)

template <int ACT>
__device__ __forceinline__ float activate(float v)
{
    if (ACT == 1) return v < 0.f ? 0.f : v;
    if (ACT == 2) return v * logistic(v);
    if (ACT == 3) {
        const float x = __builtin_fabsf(v) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * x);
        const float above = 0.5f * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f)))) * __expf(-x * x);
        return v * (v < 0.f ? above : 1.f - above);
    }
    if (ACT == kGeluF32) {
        const float u = v * v, t = __builtin_amdgcn_rcpf(1.f + 0.4f * __builtin_fabsf(v));
        const float near = 0.5f + v * (0.39894223f + u * (-0.06648978f + u * (0.0099708224f + u * (-0.0011817829f + u * (0.00010976343f + u * -6.518569e-6f)))));
        const float above = t * (0.15959956f + t * (0.15903236f + t * (0.13948295f + t * (0.053804465f + t * (0.1087361f + t * (-0.18978289f + t * 0.06946121f)))))) *
                            __builtin_amdgcn_exp2f(-0.72134752f * u);
        return v * (u < 1.5625f ? near : v < 0.f ? above : 1.f - above);
    }
    if (ACT == 4) return v * logistic(1.5957691216057308f * (v + 0.044715f * v * v * v));
    return v;
}

// (one branch for all: a branch a number is most of an epilogue's time)
template <int N>
__device__ __forceinline__ void activate_all(float (&v)[N], int act, int dtype)
{
    auto each = [&](auto f) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = f(v[e]);
    };
    if (act == 2) each([](float x) { return activate<2>(x); });
    else if (act == 4) each([](float x) { return activate<4>(x); });
    else if (act == 3 && dtype == kF32) each([](float x) { return activate<kGeluF32>(x); });
    else if (act == 3) each([](float x) { return activate<3>(x); });
    else if (act == 1) each([](float x) { return activate<1>(x); });
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

// Eight numbers of a stream of type DT: their bits, to and from float32
template <int DT>
struct Eight {
    v4i b[DT == kF32 ? 2 : 1];
};

template <int DT>
__device__ __forceinline__ Eight<DT> load_eight(const void *p, long long i)
{
    Eight<DT> r;
    if constexpr (DT == kF32) {
        r.b[0] = *(const v4i_any *)((const float *)p + i);
        r.b[1] = *(const v4i_any *)((const float *)p + i + 4);
    } else {
        r.b[0] = *(const v4i_any *)((const uint16_t *)p + i);
    }
    return r;
}

template <int DT>
__device__ __forceinline__ float value_of(const Eight<DT> &r, int e)
{
    if constexpr (DT == kF32) {
        const int w = r.b[e >> 2][e & 3];          // (a bit cast of the vector's element itself takes the first one)
        return __builtin_bit_cast(float, w);
    } else {
        const uint32_t w = (uint32_t)r.b[0][e >> 1];
        if (DT == kF16) return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> (16 * (e & 1))));
        return __builtin_bit_cast(float, e & 1 ? w & 0xffff0000u : w << 16);
    }
}

template <int DT>
__device__ __forceinline__ void store_eight(void *p, long long i, const float (&v)[8])
{
    if constexpr (DT == kF32) {
        *(v4f_any *)((float *)p + i) = v4f{v[0], v[1], v[2], v[3]};
        *(v4f_any *)((float *)p + i + 4) = v4f{v[4], v[5], v[6], v[7]};
    } else {
        v4i t;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const v2f two = {v[2 * e], v[2 * e + 1]};
            t[e] = DT == kF16 ? __builtin_bit_cast(int, __builtin_convertvector(two, v2h)) : __builtin_bit_cast(int, __builtin_convertvector(two, v2b));
        }
        *(v4i_any *)((uint16_t *)p + i) = t;
    }
}

// The same of the `left` numbers (1 to 7) that a row still has, the last one in the others' places
template <int DT>
__device__ __forceinline__ Eight<DT> load_up_to_eight(const void *p, int left)
{
    Eight<DT> r = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = load_bits(p, min(e, left - 1), DT);
        if (DT == kF32) r.b[DT == kF32 ? e >> 2 : 0][e & 3] = (int)b;
        else r.b[0][e >> 1] |= (int)(b << (16 * (e & 1)));
    }
    return r;
}

// Eight scales or biases from p[n] on
__device__ __forceinline__ void load_column(const float *p, int n, int N, float (&v)[8])
{
    const Eight<kF32> t = n + 8 <= N ? load_eight<kF32>(p, n) : load_up_to_eight<kF32>(p + n, N - n);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = value_of<kF32>(t, e);
}

// A piece of k that goes beyond a row's end is read as the row's last 16 numbers, in both operands alike, so that each still meets its own.  What is left of the row
// (16: all of them, 0 or less: none) is its last `left` numbers, the others have been in the piece before: in the rows, not the weights, they are made zeros.
__device__ __forceinline__ v4i last_of(const v4i &v, int left)
{
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int over = 16 - left - 4 * i;                // numbers of these four to clear
        r[i] = over >= 4 ? 0 : (int)((unsigned)v[i] & 0xffffffffu << (8 * max(over, 0)));
    }
    return r;
}

// Outputs n .. n + 3 of row m from their sums, one product's or two: what the kernels use that have four sums of a row in a lane.  The columns' scales and
// biases and the row's are loaded ahead (load_four), while the sums are still being taken.
template <bool GATED>
struct Four {
    float xs, s1[4], b1[4], s2[4], b2[4];
    uint32_t res[4];
};

template <bool GATED>
__device__ __forceinline__ void load_four(const LinearArgs &a, int m, int n, Four<GATED> &f)
{
    f.xs = a.xs[m];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int at = min(n + e, a.N - 1);
        f.s1[e] = a.ws[at];
        f.b1[e] = a.bias ? a.bias[at] : 0.f;
        if (GATED) {
            f.s2[e] = a.ws2[at];
            f.b2[e] = a.bias2 ? a.bias2[at] : 0.f;
        } else {
            f.res[e] = a.res ? load_bits(a.res, m * a.ldr + at, a.dtype) : 0;
        }
    }
}

template <bool GATED>
__device__ __forceinline__ void finish_four(const LinearArgs &a, const v4i &c, const v4i &c2, const Four<GATED> &f, int m, int n)
{
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)c[e] * f.xs * f.s1[e] + f.b1[e];
    activate_all(v, a.act, a.dtype);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < a.N) {
            if (GATED) v[e] *= (float)c2[e] * f.xs * f.s2[e] + f.b2[e];
            else if (a.res) v[e] += value_of(f.res[e], a.dtype);
            store_number(a.y, m * a.ldy + n + e, a.dtype, v[e]);
        }
}

}  // namespace icnn
