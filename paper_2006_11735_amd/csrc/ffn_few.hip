// The kernels of ffn_few.h for products with one set of weights.
#include "ffn_few.h"

namespace icnn {

template <int MT, bool GATED, bool DIRECT>
__global__ __launch_bounds__(NW * 64) void linear_few_kernel(const LinearArgs a)
{
    few_product<MT, GATED, DIRECT, false>(a, nullptr, (int)blockIdx.x * 16, 0);
}

template <int MT, bool GATED, bool DIRECT>
static hipError_t launch_one(const LinearArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((linear_few_kernel<MT, GATED, DIRECT>), dim3((unsigned)((a.N + 15) / 16)), dim3(NW * 64), (few_lds<MT, GATED>()), st, a);
    return hipGetLastError();
}

template <int MT>
static hipError_t launch_few(const LinearArgs &a, hipStream_t st)
{
    if (few_direct(a, 0)) return a.w2 ? launch_one<MT, true, true>(a, st) : launch_one<MT, false, true>(a, st);
    return a.w2 ? launch_one<MT, true, false>(a, st) : launch_one<MT, false, false>(a, st);
}

hipError_t launch_few_linear(const LinearArgs &a, hipStream_t st)
{
    return a.M <= 16 ? launch_few<1>(a, st) : a.M <= 32 ? launch_few<2>(a, st) : launch_few<4>(a, st);
}

}  // namespace icnn
