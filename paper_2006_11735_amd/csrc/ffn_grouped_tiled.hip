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

// Tiles of two sizes in one launch: an expert's positions in groups of 256, what is left of them in one of 256 or, up to 128, of 128; and where the tiles of 256 rows do
// not fill the chip's 256 compute units once more, those beyond the last time they do as two of 128 each, if that ends sooner.  A tile of 128 takes 0.56 of the time.
// (4096 rows, top 2 of 8, 8192 -> 4096: 316 us in tiles of one size, 285 so.)
template <bool GATED, bool DIRECT>
__global__ __launch_bounds__(512, 2) void grouped_mixed_kernel(const TiledArgs ta, const GroupedArgs ga)
{
    constexpr int BIG = 256, SMALL = 128, BN = GATED ? 128 : 256;
    const Shares shares(ga);
    const int groups = min(shares.groups<BIG, kWholeOrMost>(), ta.tiles_m), rests = min(shares.groups<BIG, kRest>(), ta.tiles_m), tiles_n = ta.tiles_n;
    int bigs = groups * tiles_n, smalls = rests * tiles_n, cut = bigs & 255;
    if (cut) {
        const int room = 256 - cut, kept = 100 + 56 * ((max(smalls - room, 0) + 255) / 256), halved = 56 * ((2 * cut + smalls + 255) / 256);
        if (halved >= kept) cut = 0;
    }
    bigs -= cut;
    smalls += 2 * cut;
    const int x = (int)(blockIdx.x & 7), i = (int)(blockIdx.x >> 3), per_big = (bigs + 7) / 8, per_small = (smalls + 7) / 8;
    const bool big = i < per_big;
    const int unit = big ? x * per_big + i : x * per_small + i - per_big;
    if (i >= per_big + per_small || unit >= (big ? bigs : smalls)) return;
    int tm, tn;
    Place p;
    if (big || unit < 2 * cut) {
        tile_at(big ? unit : bigs + unit / 2, groups, tiles_n, &tm, &tn);
        p = shares.place<BIG, kWholeOrMost>(tm);
        if (!big) p.m0 += SMALL * (unit & 1);
    } else {
        tm = (unit - 2 * cut) / tiles_n;
        tn = unit - 2 * cut - tm * tiles_n;
        p = shares.place<BIG, kRest>(tm);
    }
    if (p.expert < 0 || p.m0 >= p.end) return;
    const LinearArgs a = of_expert<GATED>(ga, p.expert, p.end);
    if (big) tiled_product<2, 4, 4, 2, 128, 2, GATED, DIRECT, true>(ta, a, &ga, tn * BN, p.m0);
    else tiled_product<2, 2, 4, 2, 128, DIRECT ? 3 : 2, GATED, DIRECT, true>(ta, a, &ga, tn * BN, p.m0);
}

template <bool GATED, bool DIRECT>
static hipError_t launch_mixed(const GroupedArgs &a, hipStream_t st)
{
    constexpr int BN = GATED ? 128 : 256, LDS = 3 * (256 + 128) * 128;
    static_assert(LDS >= 2 * (256 + 256) * 128, "either size's stages");
    TiledArgs t = {};
    t.l = a.l;
    t.tiles_n = (a.l.N + BN - 1) / BN;
    const long long groups = grouped_slots(a.l.M, a.experts, 256), per = (groups * t.tiles_n + 256) / 8 + 2;
    if (!fits_launch(per * 8, 512)) return hipErrorInvalidValue;
    t.tiles_m = (int)groups;
    t.splits = 1;
    t.steps_per = (a.l.K + 127) / 128;
    auto *const k = grouped_mixed_kernel<GATED, DIRECT>;
    if (hipError_t e = allow_large_lds((const void *)k)) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)(per * 8)), dim3(512), LDS, st, t, a);
    return hipGetLastError();
}

// (the cases in the order of kTiles, and the one of two sizes)
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
        if (tiled_direct(a.l, a.expert_stride)) return a.l.w2 ? launch_mixed<true, true>(a, st) : launch_mixed<false, true>(a, st);
        return a.l.w2 ? launch_mixed<true, false>(a, st) : launch_mixed<false, false>(a, st);
    default:
        if (a.l.w2) return launch_tiles<2, 1, 1, 2, 128, 4>(a, st);
        return tiled_direct(a.l, a.expert_stride) ? launch_one<1, 1, 2, 2, 128, 4, false, true>(a, st) : launch_one<1, 1, 2, 2, 128, 2, false, false>(a, st);
    }
}

}  // namespace icnn
