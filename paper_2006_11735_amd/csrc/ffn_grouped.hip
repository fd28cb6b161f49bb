// Products of 8-bit rows that lie in the order of their experts, each with its expert's 8-bit weights:
//   position i of expert e (offsets[e] <= i < offsets[e + 1]), r = index[i]:  acc = sum_k x[r][k] w_e[n][k] (int32, exact), v = acc * xs[r] * ws_e[n] + bias_e[n],
//   y[i][n] = act(v) or, gated, act(v) * v2.
// How many positions an expert has is known on the device alone: a launch has workgroups for the most groups of rows that there can be, each finds its own from the
// offsets, and those without one end.
#include "ffn_grouped.h"

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
__global__ __launch_bounds__(256) void grouped_plain_kernel(const GroupedArgs ga, int tiles_n, long long tiles)
{
    const long long tile = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const Place p = place_of<16>(ga, __builtin_amdgcn_readfirstlane((int)(tile / tiles_n)));
    if (p.expert < 0) return;
    const LinearArgs a = of_expert<GATED>(ga, p.expert);
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int n0 = (int)(tile % tiles_n) * 16, m = p.m0 + r, row = row_of(ga, min(m, p.end - 1));
    const int8_t *const x = a.x + max(row, 0) * a.ldx;
    const int8_t *const w = a.w + min(n0 + r, a.N - 1) * a.ldw;
    const int8_t *const w2 = GATED ? a.w2 + min(n0 + r, a.N - 1) * a.ldw : nullptr;
    v4i acc[2] = {};
    for (int k = 16 * g; k - 16 * g < a.K; k += 64) {
        const v4i xv = load_k16(x, k, a.K);
        acc[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_k16(w, k, a.K), xv, acc[0], 0, 0, 0);
        if (GATED) acc[1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_k16(w2, k, a.K), xv, acc[1], 0, 0, 0);
    }
    drain(acc);
    if (m >= p.end || row < 0) return;
    Four<GATED> f;
    load_four<GATED>(a, row, n0 + 4 * g, f);
    finish_four<GATED>(a, acc[0], acc[1], f, m, n0 + 4 * g);
}

hipError_t launch_grouped(const GroupedArgs &a, hipStream_t st)
{
    const int tiles_n = (a.l.N + 15) / 16;
    const long long tiles = grouped_slots(a.l.M, a.experts, 16) * tiles_n, blocks = (tiles + 3) / 4;
    if (a.l.w2) hipLaunchKernelGGL(grouped_plain_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, st, a, tiles_n, tiles);
    else hipLaunchKernelGGL(grouped_plain_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, a, tiles_n, tiles);
    return hipGetLastError();
}

}  // namespace icnn
