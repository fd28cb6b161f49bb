// Products of 8-bit rows that lie in the order of their experts, each with its expert's 8-bit weights:
//   position i of expert e (offsets[e] <= i < offsets[e + 1]), r = index[i]:  acc = sum_k x[r][k] w_e[n][k] (int32, exact), v = acc * xs[r] * ws_e[n] + bias_e[n],
//   y[i][n] = act(v) or, gated, act(v) * v2.
// How many positions an expert has is known on the device alone: a launch has workgroups for the most groups of rows that there can be, each finds its own from the
// offsets, and those without one end.
#include "ffn_few.h"
#include "ffn_tokens.h"

namespace icnn {

// One wave a tile of 16 x 16 outputs, operands straight from memory: any size, stride and alignment.
template <bool GATED>
__global__ __launch_bounds__(256) void grouped_plain_kernel(const GroupedArgs ga, int tiles_n, long long tiles)
{
    const long long tile = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const Place p = Shares(ga).place<16>(__builtin_amdgcn_readfirstlane((int)(tile / tiles_n)));
    if (p.expert < 0) return;
    const LinearArgs a = of_expert<GATED>(ga, p.expert, p.end);
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int n0 = (int)(tile % tiles_n) * 16, m = p.m0 + r, row = row_of(ga, min(m, a.M - 1));
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
    if (m >= a.M || row < 0) return;
    Four<GATED> f;
    load_four<GATED>(a, row, n0 + 4 * g, f);
    finish_four<GATED>(a, acc[0], acc[1], f, m, n0 + 4 * g);
}

static hipError_t launch_plain(const GroupedArgs &a, hipStream_t st)
{
    const int tiles_n = (a.l.N + 15) / 16;
    const long long tiles = grouped_slots(a.l.M, a.experts, 16) * tiles_n, blocks = (tiles + 3) / 4;
    if (a.l.w2) hipLaunchKernelGGL(grouped_plain_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, st, a, tiles_n, tiles);
    else hipLaunchKernelGGL(grouped_plain_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, a, tiles_n, tiles);
    return hipGetLastError();
}

template <int MT, bool GATED, bool DIRECT>
__global__ __launch_bounds__(NW * 64) void grouped_few_kernel(const GroupedArgs ga, int tiles_n)
{
    const Place p = Shares(ga).place<16 * MT>((int)blockIdx.x / tiles_n);
    if (p.expert < 0) return;
    few_product<MT, GATED, DIRECT, true>(of_expert<GATED>(ga, p.expert, p.end), &ga, (int)blockIdx.x % tiles_n * 16, p.m0);
}

// Position by position, each with its own pass over its expert's weights
template <int C, int KW, int OUT, bool GATED>
__global__ __launch_bounds__(64 * (KW > 4 ? KW : 4)) void grouped_tokens_kernel(const GroupedArgs ga, int blocks_n)
{
    const Place p = Shares(ga).place<1>((int)blockIdx.x / blocks_n);
    if (p.expert < 0) return;
    const int row = __builtin_amdgcn_readfirstlane(row_of(ga, p.m0));
    if (row < 0) return;
    LinearArgs a = of_expert<GATED>(ga, p.expert, 1);
    a.x += row * a.ldx;
    a.xs += row;
    a.y = (int8_t *)a.y + p.m0 * a.ldy * (a.dtype == kF32 ? 4 : 2);
    tokens_product<1, C, KW, OUT, GATED>(a, (int)blockIdx.x % blocks_n);
}

template <int MT, bool GATED, bool DIRECT>
static hipError_t launch_few_of(const GroupedArgs &a, hipStream_t st)
{
    const int tiles_n = (a.l.N + 15) / 16;
    const long long groups = grouped_slots(a.l.M, a.experts, 16 * MT) * tiles_n;
    if (!fits_launch(groups, NW * 64)) return launch_plain(a, st);             // (which has four groups of 16 x 16 outputs in a workgroup)
    hipLaunchKernelGGL((grouped_few_kernel<MT, GATED, DIRECT>), dim3((unsigned)groups), dim3(NW * 64), (few_lds<MT, GATED>()), st, a, tiles_n);
    return hipGetLastError();
}

template <int MT>
static hipError_t launch_few(const GroupedArgs &a, hipStream_t st)
{
    if (few_direct(a.l, a.expert_stride)) return a.l.w2 ? launch_few_of<MT, true, true>(a, st) : launch_few_of<MT, false, true>(a, st);
    return a.l.w2 ? launch_few_of<MT, true, false>(a, st) : launch_few_of<MT, false, false>(a, st);
}

template <int C, int KW, int OUT>
static hipError_t launch_tokens(const GroupedArgs &a, hipStream_t st)
{
    constexpr int NWT = KW > 4 ? KW : 4, HALF = OUT / 2 < 1 ? 1 : OUT / 2;
    const int per = (a.l.w2 ? HALF : OUT) * (NWT / KW), blocks_n = (a.l.N + per - 1) / per;
    const long long groups = (long long)a.l.M * blocks_n;
    if (!fits_launch(groups, 64 * NWT)) return launch_plain(a, st);
    if (a.l.w2) hipLaunchKernelGGL((grouped_tokens_kernel<C, KW, HALF, true>), dim3((unsigned)groups), dim3(64 * NWT), 0, st, a, blocks_n);
    else hipLaunchKernelGGL((grouped_tokens_kernel<C, KW, OUT, false>), dim3((unsigned)groups), dim3(64 * NWT), 0, st, a, blocks_n);
    return hipGetLastError();
}

hipError_t launch_grouped(const GroupedArgs &a, hipStream_t st)
{
    const GroupedPlan plan = plan_grouped_launch(a, linear_tuning());
    switch (plan.kernel) {
    case LinearKernel::tokens:
        if (a.l.K <= 1024) return launch_tokens<1, 1, 4>(a, st);
        if (a.l.K <= 2048) return launch_tokens<1, 2, 8>(a, st);
        if (a.l.K <= 4096) return launch_tokens<1, 4, 8>(a, st);
        if (a.l.K <= 8192) return launch_tokens<1, 8, 4>(a, st);
        if (a.l.K <= 16384) return launch_tokens<1, 16, 4>(a, st);
        return launch_tokens<2, 16, 4>(a, st);
    case LinearKernel::few: return plan.rows == 16 ? launch_few<1>(a, st) : plan.rows == 32 ? launch_few<2>(a, st) : launch_few<4>(a, st);
    case LinearKernel::tiled: return launch_grouped_tiled(a, plan.tile, st);
    case LinearKernel::plain: break;
    }
    return launch_plain(a, st);
}

}  // namespace icnn
