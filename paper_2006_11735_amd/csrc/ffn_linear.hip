// Products of 8-bit rows and 8-bit weights with a scale per row and one per output:
//   acc = sum_k x[m][k] w[n][k] (int32, exact: k <= 131071), v = acc * xs[m] * ws[n] + bias[n],
//   y[m][n] = act(v) + res[m][n], or, gated, act(v) * v2 with v2 of the second weights; rounded to the stream's type once.
// Weights are read as they are stored, [n][k] rows: both operands of the matrix instruction run along k, and the order of k is free as long as both sides
// have the same.
#include "ffn_common.h"

namespace icnn {

// Wait states between the last products and their sums' first reader (see mfma_drain in conv_common.h)
template <int N>
__device__ __forceinline__ void drain(v4i (&acc)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(acc[i]));
    asm volatile("s_nop 15\n\ts_nop 3");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(acc[i]));
}

// One wave a tile of 16 x 16 outputs, operands straight from memory: any size, stride and alignment.
template <bool GATED>
__global__ __launch_bounds__(256) void linear_plain_kernel(const LinearArgs a, int tiles_n, long long tiles)
{
    const long long tile = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int m0 = (int)(tile / tiles_n) * 16, n0 = (int)(tile % tiles_n) * 16;
    const int8_t *const x = a.x + min(m0 + r, a.M - 1) * a.ldx;
    const int8_t *const w = a.w + min(n0 + r, a.N - 1) * a.ldw;
    const int8_t *const w2 = GATED ? a.w2 + min(n0 + r, a.N - 1) * a.ldw : nullptr;
    v4i acc[2] = {};
    for (int k = 16 * g; k - 16 * g < a.K; k += 64) {
        const v4i xv = load_k16(x, k, a.K);
        acc[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_k16(w, k, a.K), xv, acc[0], 0, 0, 0);
        if (GATED) acc[1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_k16(w2, k, a.K), xv, acc[1], 0, 0, 0);
    }
    drain(acc);
    const int m = m0 + r;
    if (m >= a.M) return;
    Four<GATED> f;
    load_four<GATED>(a, m, n0 + 4 * g, f);
    finish_four<GATED>(a, acc[0], acc[1], f, m, n0 + 4 * g);
}

static hipError_t launch_range(const LinearArgs &a, hipStream_t st)
{
    const LinearPlan plan = plan_launch(a, linear_tuning());
    switch (plan.kernel) {
    case LinearKernel::tokens: return launch_tokens_linear(a, st);
    case LinearKernel::few: return launch_few_linear(a, st);
    case LinearKernel::tiled: return launch_tiled_linear(a, plan.tiles, st);
    case LinearKernel::plain: break;
    }
    const int tiles_n = (a.N + 15) / 16;
    const long long tiles = (long long)((a.M + 15) / 16) * tiles_n, blocks = (tiles + 3) / 4;
    if (a.w2) hipLaunchKernelGGL(linear_plain_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, st, a, tiles_n, tiles);
    else hipLaunchKernelGGL(linear_plain_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, a, tiles_n, tiles);
    return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs &a, hipStream_t st)
{
    return each_range(a, a.dtype == kF32 ? 4 : 2, [&](const LinearArgs &b) { return launch_range(b, st); });
}

}  // namespace icnn
