// The kernels of ffn_tiled.h for products grouped by expert.
#include "ffn_tiled.h"

namespace icnn {

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
__global__ __launch_bounds__(WN * WM * 64, waves_per_simd(WN * WM, 32 * (TN * WN + TM * WM) * BK * STAGES)) void grouped_tiled_kernel(const TiledArgs ta, const GroupedArgs ga)
{
    // (as many tiles as there are, over the chip's XCDs; ta.tiles_m: as many rows of them as there can be)
    constexpr int BM = 32 * TM * WM;
    const Shares shares(ga);
    const int tiles_m = min(shares.groups<BM, kAll>(), ta.tiles_m), per_xcd = (tiles_m * ta.tiles_n + 7) / 8, unit = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || unit >= tiles_m * ta.tiles_n) return;
    int tm, tn;
    tile_at(unit, tiles_m, ta.tiles_n, &tm, &tn);
    const Place p = shares.place<BM>(tm);
    if (p.expert < 0) return;
    tiled_product<TN, TM, WN, WM, BK, STAGES, GATED, DIRECT, true>(ta, of_expert<GATED>(ga, p.expert, p.end), &ga, tn * (32 * TN * WN / (GATED ? 2 : 1)), p.m0);
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
static hipError_t launch_one(const GroupedArgs &a, hipStream_t st)
{
    constexpr int BN = 32 * TN * WN / (GATED ? 2 : 1), BM = 32 * TM * WM, LDS = 32 * (TN * WN + TM * WM) * BK * STAGES + 8 * BM;
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

// Tiles of several sizes in one launch (see mixed_tile in ffn_plan.h)
template <bool GATED, bool DIRECT, bool EIGHTHS>
__global__ __launch_bounds__(512, 2) void grouped_mixed_kernel(const TiledArgs ta, const GroupedArgs ga)
{
    constexpr int ROWS = kMixedRows, BN = GATED ? 128 : 256, BN8 = 128;
    constexpr Groups REST = EIGHTHS ? kHalf : kRest;
    const Shares shares(ga);
    const int groups = min(shares.groups<ROWS, kWholeOrMost>(), ta.tiles_m), rests = min(shares.groups<ROWS, REST>(), ta.tiles_m);
    const int small = EIGHTHS ? min(shares.groups<ROWS, kQuarter>(), ta.tiles_m) : 0;
    const MixedTile t = mixed_tile<EIGHTHS>(groups, rests, small, ta.tiles_n, (ga.l.N + BN8 - 1) / BN8, ta.steps_per, blockIdx.x);
    if (t.rows == 0) return;
    Place p;
    if (t.from == kWholeOrMost) p = shares.place<ROWS, kWholeOrMost>(t.slot);
    else if (!EIGHTHS || t.from == REST) p = shares.place<ROWS, REST>(t.slot);
    else p = shares.place<ROWS, kQuarter>(t.slot);
    p.m0 += t.down;
    if (p.expert < 0 || p.m0 >= p.end) return;
    const LinearArgs a = of_expert<GATED>(ga, p.expert, p.end);
    if (t.rows == ROWS) tiled_product<2, 4, 4, 2, 128, 2, GATED, DIRECT, true>(ta, a, &ga, t.n * BN, p.m0);
    else if (t.rows == ROWS / 2) tiled_product<2, 2, 4, 2, 128, DIRECT ? 3 : 2, GATED, DIRECT, true>(ta, a, &ga, t.n * BN, p.m0);
    else if constexpr (EIGHTHS) tiled_product<1, 1, 4, 2, 128, DIRECT ? 6 : 2, false, DIRECT, true>(ta, a, &ga, t.n * BN8, p.m0);
}

template <bool GATED, bool DIRECT, bool EIGHTHS>
static hipError_t launch_mixed(const GroupedArgs &a, hipStream_t st)
{
    static_assert(!(GATED && EIGHTHS), "a wave of 32 weight rows has one layer's");
    constexpr int BN = GATED ? 128 : 256, LDS = 3 * (256 + 128) * 128 + 8 * 128;
    static_assert(LDS >= 2 * (256 + 256) * 128 + 8 * 256 && LDS >= 6 * (128 + 64) * 128 + 8 * 64, "any size's stages and rows");
    TiledArgs t = {};
    t.l = a.l;
    t.tiles_n = (a.l.N + BN - 1) / BN;
    const long long blocks = mixed_blocks<EIGHTHS>(a.l.M, a.experts, t.tiles_n);
    if (!fits_launch(blocks, 512)) return hipErrorInvalidValue;
    t.tiles_m = (int)grouped_slots(a.l.M, a.experts, kMixedRows);
    t.splits = 1;
    t.steps_per = (a.l.K + 127) / 128;
    auto *const k = grouped_mixed_kernel<GATED, DIRECT, EIGHTHS>;
    if (hipError_t e = allow_large_lds((const void *)k)) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(512), LDS, st, t, a);
    return hipGetLastError();
}

template <bool DIRECT>
static hipError_t launch_mixed_of(const GroupedArgs &a, hipStream_t st)
{
    if (a.l.w2) return launch_mixed<true, DIRECT, false>(a, st);
    return a.l.K > 31 * 128 ? launch_mixed<false, DIRECT, true>(a, st) : launch_mixed<false, DIRECT, false>(a, st);
}

// (the cases in the order of kTiles, and the one of several sizes)
hipError_t launch_grouped_tiled(const GroupedArgs &a, int tile, hipStream_t st)
{
    static_assert(kTileKinds == 6, "a case a tile");
    switch (tile) {
    case 0: return launch_tiles<2, 4, 4, 2, 128, 2>(a, st);
    case 1: return launch_tiles<2, 2, 4, 2, 128, 3>(a, st);
    case 2: return launch_tiles<2, 2, 2, 2, 128, 2>(a, st);
    case 3: return launch_tiles<2, 2, 2, 2, 128, 4>(a, st);
    case 4: return launch_tiles<2, 1, 2, 2, 128, 3>(a, st);
    case kMixedTiles:
        return tiled_direct(a.l, a.expert_stride) ? launch_mixed_of<true>(a, st) : launch_mixed_of<false>(a, st);
    default:
        if (tiled_direct(a.l, a.expert_stride)) return a.l.w2 ? launch_one<2, 1, 1, 2, 128, 4, true, true>(a, st) : launch_one<1, 1, 2, 2, 128, 4, false, true>(a, st);
        return a.l.w2 ? launch_one<2, 1, 1, 2, 128, 2, true, false>(a, st) : launch_one<1, 1, 2, 2, 128, 2, false, false>(a, st);
    }
}

}  // namespace icnn
