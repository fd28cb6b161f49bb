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

// What brings a row's numbers to 8 bits: 127 / max|v| as a float32 and what its rounding has left of it.  A number that is exactly between two of the 8-bit ones (half
// of the largest one is, at 63.5) has to stay there for its tie to go to the even one: by the first part alone one of ten such numbers went to its other side.
struct Factor {
    float most, rest;
};

// Below this the squares of a row may have been rounded as subnormal numbers or to zero: each is off by 2^-150 at most, 2^20 of them by 2^-130, which is
// nothing beside a sum or an eps of 2^-100.  What is below is taken again, from memory, in 64 bits: rows of numbers of 1e-15 and less, with hardly any eps.
constexpr float kLeastSquares = 0x1p-100f;

__device__ __forceinline__ bool squares_are_lost(float squares, uint32_t most, const RowsArgs &a)
{
    return squares < kLeastSquares && a.eps < kLeastSquares && __builtin_bit_cast(float, most) >= kLeast;
}

// Number i of the row as the norm takes it, once more: its own thread asks, which has stored the sum where there is one (maybe over x or the residual)
__device__ __forceinline__ float number_again(const RowsArgs &a, long long row, int i)
{
    if (a.sum) return load_number(a.sum, row * a.lds + i, a.dtype);
    const float x = load_number(a.x, row * a.ldx + i, a.dtype);
    return a.res ? round_number(x + load_number(a.res, row * a.ldr + i, a.dtype), a.dtype) : x;
}

// The sum over a row's threads, of one wave or of WAVES of them
template <int WAVES>
__device__ __forceinline__ double sum_of_row(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if constexpr (WAVES > 1) {
        __shared__ double part[WAVES];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
        for (int q = 0; q < WAVES; ++q) v += part[q];
    }
    return v;
}

// (a scale that would be infinite is NaN)
__device__ __forceinline__ float finite_or_nan(float scale) { return scale < __builtin_huge_valf() ? scale : __builtin_nanf(""); }

__device__ __forceinline__ float scale_of_wide(double squares, uint32_t most, const RowsArgs &a)
{
    return finite_or_nan((float)((double)__builtin_bit_cast(float, most) / 127 / sqrt(squares / a.c + (double)a.eps)));
}

// (factor for the numbers, scale of the row).  A row that holds NaN or an infinity, or whose squares do not add up to a finite sum: numbers 0, scale NaN.
__device__ __forceinline__ void row_scale(float squares, uint32_t most, const RowsArgs &a, Factor *factor, float *scale)
{
    const float m = __builtin_bit_cast(float, most);
    *factor = {};
    if (most >= 0x7f800000u || !(squares < __builtin_huge_valf())) {
        *scale = __builtin_nanf("");
    } else if (m < kLeast) {
        *scale = 0.f;
    } else {
        factor->most = 127.f / m;
        factor->rest = __builtin_fmaf(-factor->most, m, 127.f) * (factor->most * (1.f / 127.f));      // (what is left of 127, over m)
        *scale = finite_or_nan(m / 127.f * (a.gamma ? 1.f / sqrtf(squares / (float)a.c + a.eps) : 1.f));
    }
}

// one number in 8 bits; a factor of 0 makes any number 0
__device__ __forceinline__ int to_byte(float v, const Factor &f)
{
    return f.most == 0.f ? 0 : (int)rintf(__builtin_fmaf(v, f.most, v * f.rest));
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
    Factor factor;
    float scale;
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
    if (a.gamma && squares_are_lost(squares, most, a)) {
        double wide = 0;
        for (int i = t; i < a.c; i += 256) {
            const double s = number_again(a, row, i);
            wide += s * s;
        }
        scale = scale_of_wide(sum_of_row<4>(wide), most, a);
        if (t == 0) a.scale[row] = scale;
    }
}

// Eight numbers of a stream that is read once
template <int DT>
__device__ __forceinline__ Eight<DT> stream_eight(const void *p, long long i)
{
    Eight<DT> r;
    if constexpr (DT == kF32) {
        r.b[0] = __builtin_nontemporal_load((const v4i_any *)((const float *)p + i));
        r.b[1] = __builtin_nontemporal_load((const v4i_any *)((const float *)p + i + 4));
    } else {
        r.b[0] = __builtin_nontemporal_load((const v4i_any *)((const uint16_t *)p + i));
    }
    return r;
}

typedef int v2i_any __attribute__((ext_vector_type(2), aligned(1)));

// Rows that fit a workgroup's registers: read once.  T threads a row (a wave, with neither LDS nor a barrier, or more), V times eight numbers a thread.  All loads of a
// row are on their way before the first is waited for: they stay bits until then, since a conversion in the branch that has loaded would wait there.
// DT: the stream's type; GT: gamma's, 0 = no norm; TINY: eps is so small that squares may be lost (1 x 4096 2.9 us, with the code for them 3.0).
template <int DT, int GT, bool TINY, int T, int V>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rows_held_kernel(const RowsArgs a)
{
    constexpr int WAVES = T / 64, GD = GT ? GT : kF32;
    const long long row = T < 256 ? (long long)blockIdx.x * (256 / T) + threadIdx.x / T : (long long)blockIdx.x;
    const int t = threadIdx.x % T;
    if (T < 256 && row >= a.rows) return;
    Eight<DT> x[V], r[V];
    Eight<GD> gm[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int i = 8 * (k * T + t);
        x[k] = {};
        if (i + 8 <= a.c) x[k] = stream_eight<DT>(a.x, row * a.ldx + i);
        else if (i < a.c) x[k] = load_up_to_eight<DT>((const uint8_t *)a.x + (row * a.ldx + i) * (DT == kF32 ? 4 : 2), a.c - i);
    }
    if (GT && a.res) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int i = 8 * (k * T + t);
            r[k] = {};
            if (i + 8 <= a.c) r[k] = stream_eight<DT>(a.res, row * a.ldr + i);
            else if (i < a.c) r[k] = load_up_to_eight<DT>((const uint8_t *)a.res + (row * a.ldr + i) * (DT == kF32 ? 4 : 2), a.c - i);
        }
    }
    if (GT) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int i = 8 * (k * T + t);
            gm[k] = {};
            if (i + 8 <= a.c) gm[k] = load_eight<GD>(a.gamma, i);
            else if (i < a.c) gm[k] = load_up_to_eight<GD>((const uint8_t *)a.gamma + i * (GD == kF32 ? 4 : 2), a.c - i);
        }
    }
    float v[V][8], squares = 0.f;
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int i = 8 * (k * T + t), left = a.c - i;                     // (numbers behind the row's end repeat its last one: they do not count)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] = value_of<DT>(x[k], e);
        if (GT && a.res) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = round_number(v[k][e] + value_of<DT>(r[k], e), DT);
        }
        if (GT && a.sum) {
            uint8_t *const at = (uint8_t *)a.sum + (row * a.lds + i) * (DT == kF32 ? 4 : 2);
            if (left >= 8) {
                store_eight<DT>(at, 0, v[k]);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < left) store_number(at, e, DT, v[k][e]);
            }
        }
        if (left < 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = e < left ? v[k][e] : 0.f;
        }
        if (GT) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                squares += v[k][e] * v[k][e];
                v[k][e] *= value_of<GD>(gm[k], e);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[k][e]));
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        if (GT) squares += __shfl_xor(squares, d);
        most = max(most, (uint32_t)__shfl_xor((int)most, d));
    }
    if constexpr (WAVES > 1) {
        __shared__ float squares_of[WAVES];
        __shared__ uint32_t most_of[WAVES];
        if ((t & 63) == 0) {
            squares_of[t >> 6] = squares;
            most_of[t >> 6] = most;
        }
        __syncthreads();
        squares = 0.f;
#pragma unroll
        for (int q = 0; q < WAVES; ++q) {
            squares += squares_of[q];
            most = max(most, most_of[q]);
        }
    }
    Factor factor;
    float scale;
    row_scale(squares, most, a, &factor, &scale);
    if (t == 0) a.scale[row] = scale;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int i = 8 * (k * T + t);
        uint32_t b[2] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e >> 2] |= (uint32_t)(to_byte(v[k][e], factor) & 255) << (8 * (e & 3));
        int8_t *const at = a.q + row * a.ldq + i;
        if (i + 8 <= a.c) {
            *(v2i_any *)at = v2i_any{(int)b[0], (int)b[1]};
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (i + e < a.c) at[e] = (int8_t)(b[e >> 2] >> (8 * (e & 3)));
        }
    }
    if (TINY && squares_are_lost(squares, most, a)) {
        double wide = 0;
        for (int k = 0; k < V; ++k)
            for (int i = 8 * (k * T + t), e = 0; e < 8 && i + e < a.c; ++e) {
                const double s = number_again(a, row, i + e);
                wide += s * s;
            }
        scale = scale_of_wide(sum_of_row<WAVES>(wide), most, a);
        if (t == 0) a.scale[row] = scale;
    }
}

template <int DT, int GT, bool TINY>
static hipError_t launch_rows_held(const RowsArgs &a, hipStream_t st)
{
    const dim3 four((unsigned)((a.rows + 3) / 4)), one((unsigned)a.rows);
    if (a.c <= 512) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 64, 1>), four, dim3(256), 0, st, a);
    else if (a.c <= 1024) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 64, 2>), four, dim3(256), 0, st, a);
    else if (a.c <= 2048) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 256, 1>), one, dim3(256), 0, st, a);
    else if (a.c <= 4096) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 256, 2>), one, dim3(256), 0, st, a);
    else if (a.c <= 6144) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 256, 3>), one, dim3(256), 0, st, a);
    else if (a.c <= 8192) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 256, 4>), one, dim3(256), 0, st, a);
    else if (a.c <= 16384) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 512, 4>), one, dim3(512), 0, st, a);      // (by 1024 threads: 2048 x 16384 20.6 us instead of 18.7, 2048 x 11008 18.1 instead of 15)
    else if (a.c <= 32768) hipLaunchKernelGGL((rows_held_kernel<DT, GT, TINY, 1024, 4>), one, dim3(1024), 0, st, a);
    else hipLaunchKernelGGL(rows_kernel, one, dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int DT, int GT>
static hipError_t launch_rows_of(const RowsArgs &a, hipStream_t st)
{
    if constexpr (GT != 0)
        if (a.eps < kLeastSquares) return launch_rows_held<DT, GT, true>(a, st);
    return launch_rows_held<DT, GT, false>(a, st);
}

static hipError_t launch_some_rows(const RowsArgs &a, hipStream_t st)
{
    const bool f32_gamma = a.gamma_dtype == kF32;
    if (!a.gamma) return a.dtype == kF32 ? launch_rows_of<kF32, 0>(a, st) : a.dtype == kF16 ? launch_rows_of<kF16, 0>(a, st) : launch_rows_of<kBf16, 0>(a, st);
    if (a.dtype == kF32) return launch_rows_of<kF32, kF32>(a, st);
    if (a.dtype == kF16) return f32_gamma ? launch_rows_of<kF16, kF32>(a, st) : launch_rows_of<kF16, kF16>(a, st);
    return f32_gamma ? launch_rows_of<kBf16, kF32>(a, st) : launch_rows_of<kBf16, kBf16>(a, st);
}

// (rows that one launch does not hold go in several)
hipError_t launch_rows(const RowsArgs &a, hipStream_t st)
{
    constexpr long long MOST = 1 << 21;
    static_assert(fits_launch(MOST, 1024), "a workgroup a row");
    const int item = a.dtype == kF32 ? 4 : 2;
    for (long long at = 0; at < a.rows; at += MOST) {
        RowsArgs b = a;
        b.rows = a.rows - at < MOST ? a.rows - at : MOST;
        b.x = (const uint8_t *)a.x + at * a.ldx * item;
        if (a.res) b.res = (const uint8_t *)a.res + at * a.ldr * item;
        if (a.sum) b.sum = (uint8_t *)a.sum + at * a.lds * item;
        b.q = a.q + at * a.ldq;
        b.scale = a.scale + at;
        if (hipError_t e = launch_some_rows(b, st)) return e;
    }
    return hipSuccess;
}

}  // namespace icnn
