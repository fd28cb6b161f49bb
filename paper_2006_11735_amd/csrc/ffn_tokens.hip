// The kernels of ffn_tokens.h for products with one set of weights.
#include "ffn_tokens.h"

namespace icnn {

template <int MR, int C, int KW, int OUT, bool GATED>
__global__ __launch_bounds__(64 * (KW > 4 ? KW : 4)) void linear_tokens_kernel(const LinearArgs a)
{
    tokens_product<MR, C, KW, OUT, GATED>(a, (int)blockIdx.x);
}

template <int MR, int C, int KW, int OUT>
static void launch_tokens(const LinearArgs &a, hipStream_t st)
{
    constexpr int NW = KW > 4 ? KW : 4;
    const dim3 grid((unsigned)((a.N + OUT * (NW / KW) - 1) / (OUT * (NW / KW)))), block(64 * NW);
    if (a.w2) {
        constexpr int HALF = OUT / 2 < 1 ? 1 : OUT / 2;
        const dim3 wide((unsigned)((a.N + HALF * (NW / KW) - 1) / (HALF * (NW / KW))));
        hipLaunchKernelGGL((linear_tokens_kernel<MR, C, KW, HALF, true>), wide, block, 0, st, a);
    } else {
        hipLaunchKernelGGL((linear_tokens_kernel<MR, C, KW, OUT, false>), grid, block, 0, st, a);
    }
}

// A kilobyte of k a wave, the waves of a workgroup along k: by fewer waves with more of a row each 1 x 4096 -> 16384 takes 12.3 us instead of 11.7, 4 x 4096 ->
// 16384 14.6 instead of 12.9, 4 x 32768 -> 2048 18 instead of 14.4
template <int MR>
static void launch_rows_of(const LinearArgs &a, hipStream_t st)
{
    if (a.K <= 1024) launch_tokens<MR, 1, 1, 4>(a, st);
    else if (a.K <= 2048) launch_tokens<MR, 1, 2, 8>(a, st);
    else if (a.K <= 4096) launch_tokens<MR, 1, 4, 8>(a, st);
    else if (a.K <= 8192) launch_tokens<MR, 1, 8, 4>(a, st);
    else if (a.K <= 16384) launch_tokens<MR, 1, 16, 4>(a, st);
    else launch_tokens<MR, 2, 16, 4>(a, st);
}

hipError_t launch_tokens_linear(const LinearArgs &a, hipStream_t st)
{
    if (a.M == 1) launch_rows_of<1>(a, st);
    else if (a.M == 2) launch_rows_of<2>(a, st);
    else launch_rows_of<4>(a, st);
    return hipGetLastError();
}

}  // namespace icnn
