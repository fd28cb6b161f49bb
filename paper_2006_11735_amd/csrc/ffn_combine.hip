// The sum of a token's expert rows by its gates, on top of the stream: y[t] = residual[t] + sum over j of gate[t][j] v[place[t][j]], in float32, rounded once.
// Bound by the rows' way through memory: each is read once, eight numbers a lane, past the caches (4096 x 4096, top 4, in float16, on operands that no cache
// holds, 36.7 us, 5.5 TB/s; loads that keep them 39; the same operands again 32.6 us).
#include "ffn_common.h"

#include <type_traits>

namespace icnn {

// A thread has eight columns of a row; rows and columns in strides of the grid.  Four choices' rows are on their way at a time: the loads hang on no condition (a choice
// that names no row reads row 0 and counts for nothing), since behind a branch the compiler waits for each.
template <int DT, int VT>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a, int pieces, long long units)
{
    constexpr int AT_ONCE = 4;
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < units; u += (long long)gridDim.x * 256) {
        const long long t = u / pieces;
        const int c = (int)(u - t * pieces) * 8, left = a.c - c;
        const int32_t *const place = a.place + t * a.top;
        const float *const gate = a.gate + t * a.top;
        auto row = [&](auto whole) {
            Eight<DT> r = {};
            if (a.res) {
                const long long at = t * a.ldr + c;
                r = whole ? load_eight<DT>(a.res, at) : load_up_to_eight<DT>((const uint8_t *)a.res + at * (DT == kF32 ? 4 : 2), left);
            }
            float sum[8] = {};
            for (int j0 = 0; j0 < a.top; j0 += AT_ONCE) {
                int p[AT_ONCE];
                float g[AT_ONCE];
                Eight<VT> v[AT_ONCE];
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    p[j] = place[min(j0 + j, a.top - 1)];
                    g[j] = gate[min(j0 + j, a.top - 1)];
                }
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    if (j0 + j >= a.top || p[j] < 0 || p[j] >= a.v_rows) p[j] = -1;
                    const long long at = max(p[j], 0) * a.ldv + c;
                    v[j] = whole ? load_eight_once<VT>(a.v, at) : load_up_to_eight<VT>((const uint8_t *)a.v + at * (VT == kF32 ? 4 : 2), left);
                }
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] = p[j] >= 0 ? sum[e] + g[j] * value_of<VT>(v[j], e) : sum[e];
            }
            if (a.res) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += value_of<DT>(r, e);
            }
            if (whole) {
                store_eight<DT>(a.y, t * a.ldy + c, sum);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < left) store_number(a.y, t * a.ldy + c + e, DT, sum[e]);
            }
        };
        if (left >= 8) row(std::true_type{});
        else row(std::false_type{});
    }
}

template <int DT>
static hipError_t launch_of(const CombineArgs &a, hipStream_t st)
{
    const int pieces = (a.c + 7) / 8;
    const long long units = a.rows * pieces, blocks = (units + 255) / 256;
    const dim3 grid((unsigned)(blocks < (1 << 22) ? blocks : 1 << 22));
    if (a.v_dtype == kF32) hipLaunchKernelGGL((combine_kernel<DT, kF32>), grid, dim3(256), 0, st, a, pieces, units);
    else if (a.v_dtype == kF16) hipLaunchKernelGGL((combine_kernel<DT, kF16>), grid, dim3(256), 0, st, a, pieces, units);
    else hipLaunchKernelGGL((combine_kernel<DT, kBf16>), grid, dim3(256), 0, st, a, pieces, units);
    return hipGetLastError();
}

hipError_t launch_combine(const CombineArgs &args, hipStream_t st)
{
    CombineArgs a = args;
    if (a.v_rows == 0) a.top = 0;                          // (no row to read)
    return a.dtype == kF32 ? launch_of<kF32>(a, st) : a.dtype == kF16 ? launch_of<kF16>(a, st) : launch_of<kBf16>(a, st);
}

}  // namespace icnn
