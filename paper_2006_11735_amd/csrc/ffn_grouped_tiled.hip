// The kernels of ffn_tiled.h for products grouped by expert.
#include "ffn_tiled.h"

namespace icnn {

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
__global__ __launch_bounds__(WN * WM * 64, waves_per_simd(WN * WM, 32 * (TN * WN + TM * WM) * BK * STAGES)) void grouped_tiled_kernel(const TiledArgs ta, const GroupedArgs ga)
{
    tiled_product<TN, TM, WN, WM, BK, STAGES, GATED, DIRECT, true>(ta, &ga);
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
static hipError_t launch_one(const GroupedArgs &a, hipStream_t st)
{
    constexpr int BN = 32 * TN * WN / (GATED ? 2 : 1), BM = 32 * TM * WM, LDS = 32 * (TN * WN + TM * WM) * BK * STAGES;
    TiledArgs t = {};
    t.l = a.l;
    t.tiles_n = (a.l.N + BN - 1) / BN;
    const long long groups = grouped_slots(a.l.M, a.experts, BM), per = (groups * t.tiles_n + 7) / 8;
    if (!fits_launch(per * 8, WN * WM * 64)) return hipErrorInvalidValue;
    t.tiles_m = (int)groups;
    t.splits = 1;
    t.steps_per = (a.l.K + BK - 1) / BK;
    auto *const k = grouped_tiled_kernel<TN, TM, WN, WM, BK, STAGES, GATED, DIRECT>;
    if (LDS > 65536)
        if (hipError_t e = allow_large_lds((const void *)k)) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)(per * 8)), dim3(WN * WM * 64), LDS, st, t, a);
    return hipGetLastError();
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES>
static hipError_t launch_tiles(const GroupedArgs &a, hipStream_t st)
{
    if (tiled_direct(a.l, a.expert_stride))
        return a.l.w2 ? launch_one<TN, TM, WN, WM, BK, STAGES, true, true>(a, st) : launch_one<TN, TM, WN, WM, BK, STAGES, false, true>(a, st);
    return a.l.w2 ? launch_one<TN, TM, WN, WM, BK, 2, true, false>(a, st) : launch_one<TN, TM, WN, WM, BK, 2, false, false>(a, st);
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES>
static hipError_t launch_direct(const GroupedArgs &a, hipStream_t st)
{
    if (!tiled_direct(a.l, a.expert_stride)) return launch_tiles<2, 2, 4, 2, 128, 3>(a, st);
    return a.l.w2 ? launch_one<TN, TM, WN, WM, BK, STAGES, true, true>(a, st) : launch_one<TN, TM, WN, WM, BK, STAGES, false, true>(a, st);
}

// (the cases in the order of kTiles)
hipError_t launch_grouped_tiled(const GroupedArgs &a, int tile, hipStream_t st)
{
    static_assert(kTileKinds == 6, "a case a tile");
    switch (tile) {
    case 0: return launch_tiles<2, 4, 4, 2, 128, 2>(a, st);
    case 1: return launch_tiles<2, 2, 4, 2, 128, 3>(a, st);
    case 2: return launch_tiles<2, 2, 2, 2, 128, 2>(a, st);
    case 3: return launch_tiles<2, 2, 2, 2, 128, 4>(a, st);
    case 4: return launch_tiles<2, 1, 2, 2, 128, 3>(a, st);
    case 6: return launch_direct<4, 2, 2, 2, 64, 3>(a, st);
    case 7: return launch_direct<2, 4, 2, 2, 64, 3>(a, st);
    case 8: return launch_direct<2, 2, 2, 2, 64, 4>(a, st);
    default:
        if (a.l.w2) return launch_tiles<2, 1, 1, 2, 128, 4>(a, st);
        return tiled_direct(a.l, a.expert_stride) ? launch_one<1, 1, 2, 2, 128, 4, false, true>(a, st) : launch_one<1, 1, 2, 2, 128, 2, false, false>(a, st);
    }
}

}  // namespace icnn
