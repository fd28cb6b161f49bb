// The sum of a token's expert rows by its gates, on top of the stream: y[t] = residual[t] + sum over j of gate[t][j] v[place[t][j]], in float32, rounded once.
// Bound by the rows' way through memory: each is read once, eight numbers a lane.
#include "ffn_common.h"

#include <type_traits>

namespace icnn {

// A thread has eight columns of a row; rows and columns in strides of the grid.
template <int DT, int VT>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a, int pieces, long long units)
{
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < units; u += (long long)gridDim.x * 256) {
        const long long t = u / pieces;
        const int c = (int)(u - t * pieces) * 8, left = a.c - c;
        float sum[8] = {};
        for (int j = 0; j < a.top; ++j) {
            const int p = a.place[t * a.top + j];
            const float g = a.gate[t * a.top + j];
            if (p < 0 || p >= a.v_rows) continue;
            const long long at = p * a.ldv + c;
            const Eight<VT> v = left >= 8 ? load_eight<VT>(a.v, at) : load_up_to_eight<VT>((const uint8_t *)a.v + at * (VT == kF32 ? 4 : 2), left);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += g * value_of<VT>(v, e);
        }
        if (a.res) {
            const long long at = t * a.ldr + c;
            const Eight<DT> r = left >= 8 ? load_eight<DT>(a.res, at) : load_up_to_eight<DT>((const uint8_t *)a.res + at * (DT == kF32 ? 4 : 2), left);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += value_of<DT>(r, e);
        }
        if (left >= 8) {
            store_eight<DT>(a.y, t * a.ldy + c, sum);
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) store_number(a.y, t * a.ldy + c + e, DT, sum[e]);
        }
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

hipError_t launch_combine(const CombineArgs &a, hipStream_t st)
{
    return a.dtype == kF32 ? launch_of<kF32>(a, st) : a.dtype == kF16 ? launch_of<kF16>(a, st) : launch_of<kBf16>(a, st);
}

}  // namespace icnn
