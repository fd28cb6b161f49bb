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

// Tiles of several sizes in one launch: an expert's positions in groups of 256, what is left of them in one of 256 or, up to 128 or 64, of so many.  Where the tiles of
// 256 x 256 do not fill the chip's 256 compute units once more, those beyond the last time they do may be cut in two of 128 x 256 or in eight of 64 x 128, and so may the
// rests' tiles of 128 x 256 in four: whatever is expected to end soonest.  In hundredths of a tile's time half of it takes 56 and an eighth `eighth` (8192 -> 8192: 37 us of
// 163, 1024 -> 8192 12 of 33).  EIGHTHS: from 32 steps of k on (2048 rows, top 2 of 8, 4096 -> 4096 103 us without, 97 with; 4096, top 4 of 32, 2048 -> 2048 108 and 111), but
// not in gated layers, where a wave needs both layers' rows: 64 rows take 40 there (2048, top 4 of 32, 2048 -> 2048 107 and 113; 98 to 110 by now).
// (4096 rows, top 2 of 8, 8192 -> 4096: 316 us in tiles of one size, 304 in two, 289 in three; the latter 276 to 286 by now.)
constexpr int kMostCut = 1024;     // workgroups that cuts may add

template <bool GATED, bool DIRECT, bool EIGHTHS>
__global__ __launch_bounds__(512, 2) void grouped_mixed_kernel(const TiledArgs ta, const GroupedArgs ga)
{
    constexpr int ROWS = 256, BN = GATED ? 128 : 256, BN8 = 128, PARTS = 8, HALF = 56;
    constexpr Groups REST = EIGHTHS ? kHalf : kRest;
    const Shares shares(ga);
    const int groups = min(shares.groups<ROWS, kWholeOrMost>(), ta.tiles_m), tiles_n = ta.tiles_n, tiles8_n = (ga.l.N + BN8 - 1) / BN8, eighth = 22 + 120 / ta.steps_per;
    const int whole = groups * tiles_n, rests = min(shares.groups<ROWS, REST>(), ta.tiles_m) * tiles_n, beyond = whole & 255;
    const int small = EIGHTHS ? min(shares.groups<ROWS, kQuarter>(), ta.tiles_m) * tiles8_n : 0;
    // Of the tiles beyond the last full turn `in2` are cut in halves or `in8` in eighths, of the rests' halves `in4` in quarters
    int in2 = 0, in8 = 0, in4 = 0, least = 0x7fffffff;
    auto option = [&](int h, int e, int r) {
        if (h + e * (PARTS - 1) + r * (PARTS / 2 - 1) > kMostCut) return;
        const int bigs = beyond - h - e, halves = rests + 2 * h - r, eighths = small + e * PARTS + r * (PARTS / 2), room = 256 - bigs;
        const int first = bigs ? 100 : 0, then = halves ? max(first, HALF) + HALF * ((max(halves - room, 0) + 255) / 256) : first;
        const int end = max(then, (100 * bigs + HALF * halves + eighth * eighths) / 256 + (eighths ? eighth / 2 : 0));
        if (end < least) {
            least = end;
            in2 = h;
            in8 = e;
            in4 = r;
        }
    };
    option(0, 0, 0);
    option(beyond, 0, 0);
    if (EIGHTHS) {
        option(0, beyond, 0);
        option(0, beyond, rests);
        option(beyond, 0, rests);
    }
    const int bigs = whole - in2 - in8, halves = rests + 2 * in2 - in4, eighths = small + in8 * PARTS + in4 * (PARTS / 2);
    const int x = (int)(blockIdx.x & 7), per_big = (bigs + 7) / 8, per_half = (halves + 7) / 8, per_eighth = (eighths + 7) / 8;
    const int i = (int)(blockIdx.x >> 3), i2 = i - per_big, i8 = i2 - per_half;
    int tm, tn;
    Place p;
    auto tile_of = [&](int tile) {
        tile_at(tile, groups, tiles_n, &tm, &tn);
        p = shares.place<ROWS, kWholeOrMost>(tm);
    };
    auto rest_of = [&](int tile) {
        tm = tile / tiles_n;
        tn = tile - tm * tiles_n;
        p = shares.place<ROWS, REST>(tm);
    };
    if (i2 < 0) {
        const int unit = x * per_big + i;
        if (unit >= bigs) return;
        tile_of(unit);
    } else if (i8 < 0) {
        const int unit = x * per_half + i2;
        if (unit >= halves) return;
        if (unit < 2 * in2) {
            tile_of(bigs + unit / 2);
            p.m0 += ROWS / 2 * (unit & 1);
        } else {
            rest_of(unit - 2 * in2);
        }
    } else if (EIGHTHS) {
        const int unit = x * per_eighth + i8, of_rests = unit - in8 * PARTS, of_small = of_rests - in4 * (PARTS / 2);
        if (i8 >= per_eighth || unit >= eighths) return;
        if (of_small < 0) {                                // 64 rows and half the columns of a tile
            const int part = of_rests < 0 ? unit % PARTS : of_rests % (PARTS / 2);
            if (of_rests < 0) tile_of(bigs + unit / PARTS);
            else rest_of(of_rests / (PARTS / 2));
            p.m0 += ROWS / 4 * (part / 2);
            tn = 2 * tn + part % 2;
        } else {
            tm = of_small / tiles8_n;
            tn = of_small - tm * tiles8_n;
            p = shares.place<ROWS, kQuarter>(tm);
        }
    }
    if ((!EIGHTHS && i8 >= 0) || p.expert < 0 || p.m0 >= p.end || (i8 >= 0 && tn >= tiles8_n)) return;
    const LinearArgs a = of_expert<GATED>(ga, p.expert, p.end);
    if (i2 < 0) tiled_product<2, 4, 4, 2, 128, 2, GATED, DIRECT, true>(ta, a, &ga, tn * BN, p.m0);
    else if (i8 < 0) tiled_product<2, 2, 4, 2, 128, DIRECT ? 3 : 2, GATED, DIRECT, true>(ta, a, &ga, tn * BN, p.m0);
    else if constexpr (EIGHTHS) tiled_product<1, 1, 4, 2, 128, DIRECT ? 6 : 2, false, DIRECT, true>(ta, a, &ga, tn * BN8, p.m0);
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
    // (a group's tiles, or twice as many of a rest's; what cuts add; up to 7 / 8 of a workgroup for each XCD and size)
    const long long groups = grouped_slots(a.l.M, a.experts, 256), rests = groups - a.l.M / 256;
    const long long per = ((EIGHTHS ? groups + rests : groups) * t.tiles_n + (EIGHTHS ? kMostCut : 256)) / 8 + 4;
    if (!fits_launch(per * 8, 512)) return hipErrorInvalidValue;
    t.tiles_m = (int)groups;
    t.splits = 1;
    t.steps_per = (a.l.K + 127) / 128;
    auto *const k = grouped_mixed_kernel<GATED, DIRECT, EIGHTHS>;
    if (hipError_t e = allow_large_lds((const void *)k)) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)(per * 8)), dim3(512), LDS, st, t, a);
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
        if (a.l.w2) return launch_tiles<2, 1, 1, 2, 128, 4>(a, st);
        return tiled_direct(a.l, a.expert_stride) ? launch_one<1, 1, 2, 2, 128, 4, false, true>(a, st) : launch_one<1, 1, 2, 2, 128, 2, false, false>(a, st);
    }
}

}  // namespace icnn
