// The kernels of ffn_tiled.h for products with one set of weights.
#include "ffn_tiled.h"

namespace icnn {

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
__global__ __launch_bounds__(WN * WM * 64, waves_per_simd(WN * WM, 32 * (TN * WN + TM * WM) * BK * STAGES)) void linear_tiled_kernel(const TiledArgs ta)
{
    tiled_product<TN, TM, WN, WM, BK, STAGES, GATED, DIRECT, false>(ta, ta.l, nullptr, 0, 0);
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
static hipError_t launch_one(const LinearArgs &a, int splits, hipStream_t st)
{
    constexpr int BN = 32 * TN * WN / (GATED ? 2 : 1), BM = 32 * TM * WM, LDS = 32 * (TN * WN + TM * WM) * BK * STAGES;
    TiledArgs t;
    t.l = a;
    t.tiles_n = (a.N + BN - 1) / BN;
    t.tiles_m = (a.M + BM - 1) / BM;
    const int steps = (a.K + BK - 1) / BK;
    t.steps_per = (steps + splits - 1) / splits;
    t.splits = (steps + t.steps_per - 1) / t.steps_per;    // (no range without a step)
    t.counters = (unsigned *)a.workspace;
    t.part = (int32_t *)((uint8_t *)a.workspace + kSplitCounterBytes);
    const long long units = (long long)t.tiles_n * t.tiles_m * t.splits, per = (units + 7) / 8;
    t.per_xcd = (int)per;
    auto *const k = linear_tiled_kernel<TN, TM, WN, WM, BK, STAGES, GATED, DIRECT>;
    if (LDS > 65536)
        if (hipError_t e = allow_large_lds((const void *)k)) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)(per * 8)), dim3(WN * WM * 64), LDS, st, t);
    return hipGetLastError();
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES>
static hipError_t launch_tiles(const LinearArgs &a, int splits, hipStream_t st)
{
    if (tiled_direct(a, 0))
        return a.w2 ? launch_one<TN, TM, WN, WM, BK, STAGES, true, true>(a, splits, st) : launch_one<TN, TM, WN, WM, BK, STAGES, false, true>(a, splits, st);
    return a.w2 ? launch_one<TN, TM, WN, WM, BK, 2, true, false>(a, splits, st) : launch_one<TN, TM, WN, WM, BK, 2, false, false>(a, splits, st);
}

// (the cases in the order of kTiles)
hipError_t launch_tiled_linear(const LinearArgs &a, const TilePlan &p, hipStream_t st)
{
    static_assert(kTileKinds == 6 && kSplitCounterBytes == kWsCounterBytes, "a case a tile; counters as in the other workspaces");
    switch (p.tile) {
    case 0: return launch_tiles<2, 4, 4, 2, 128, 2>(a, p.splits, st);
    case 1: return launch_tiles<2, 2, 4, 2, 128, 3>(a, p.splits, st);
    case 2: return launch_tiles<2, 2, 2, 2, 128, 2>(a, p.splits, st);
    case 3: return launch_tiles<2, 2, 2, 2, 128, 4>(a, p.splits, st);
    case 4: return launch_tiles<2, 1, 2, 2, 128, 3>(a, p.splits, st);
    default:                                               // (four waves where gate and up need not be in one: 24 x 256 -> 8192 3.6 us, by two waves 4.2)
        if (tiled_direct(a, 0)) return a.w2 ? launch_one<2, 1, 1, 2, 128, 4, true, true>(a, p.splits, st) : launch_one<1, 1, 2, 2, 128, 4, false, true>(a, p.splits, st);
        return a.w2 ? launch_one<2, 1, 1, 2, 128, 2, true, false>(a, p.splits, st) : launch_one<1, 1, 2, 2, 128, 2, false, false>(a, p.splits, st);
    }
}

}  // namespace icnn
