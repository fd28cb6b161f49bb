// How products grouped by expert and those with 4-bit weights are launched (csrc/ffn_plan.h), by itself, for tests without a GPU.
#include "../paper_2006_11735_amd/csrc/ffn_plan.h"

#include <algorithm>
#include <vector>

using namespace icnn;

static GroupedArgs grouped_of(const long long *size, bool gated, bool index)
{
    GroupedArgs a = {};
    a.l.M = (int)size[0];
    a.x_rows = size[1];
    a.l.K = (int)size[2];
    a.l.N = (int)size[3];
    a.experts = (int)size[4];
    a.l.ldx = size[5];
    a.l.ldw = size[6];
    a.expert_stride = size[7];
    a.l.x = (const int8_t *)size[8];
    a.l.w = (const int8_t *)size[9];
    a.l.w2 = gated ? (const int8_t *)size[10] : nullptr;
    a.index = index ? (const int32_t *)16 : nullptr;
    return a;
}

// Of positions, x_rows, k, n, experts, x_stride, w_stride, expert_stride and the addresses of x, w and w_up: {kernel, tile, whether such sizes are taken, threads of the
// launch, whether it fits and so is not the plain kernel's}
extern "C" void ff_grouped(const long long *size, int gated, int index, int kernel, unsigned long long *out)
{
    const GroupedArgs a = grouped_of(size, gated, index);
    const GroupedPlan p = plan_grouped_launch(a, LinearTuning{kernel, 0});
    const unsigned long long m = (unsigned long long)a.l.M, n = (unsigned long long)a.l.N, wide = (gated ? 2 : 1) * n;
    auto slots = [&](int rows) { return (unsigned long long)grouped_slots(a.l.M, a.experts, rows); };
    unsigned long long threads = 0;
    switch (p.kernel) {
    case LinearKernel::tokens: {
        // (waves of a workgroup, waves along k, outputs a wave)
        const int k = a.l.K, along = k <= 1024 ? 1 : k <= 2048 ? 2 : k <= 4096 ? 4 : k <= 8192 ? 8 : 16, of = k > 1024 && k <= 4096 ? 8 : 4, waves = std::max(along, 4);
        const unsigned long long per = (unsigned long long)(gated ? of / 2 : of) * (waves / along);
        threads = m * ((n + per - 1) / per) * 64 * waves;
        break;
    }
    case LinearKernel::few: threads = slots(p.rows) * ((n + 15) / 16) * 256; break;
    case LinearKernel::tiled: {
        if (p.tile == kMixedTiles) {
            const int columns = gated ? 128 : 256, tiles_n = (int)((n + columns - 1) / columns);
            threads = (unsigned long long)std::max(mixed_blocks<false>(a.l.M, a.experts, tiles_n), gated ? 0 : mixed_blocks<true>(a.l.M, a.experts, tiles_n)) * 512;
            break;
        }
        const TileCost &t = kTiles[p.tile];
        threads = (slots(t.m) * ((wide + t.n - 1) / t.n) + 7) / 8 * 8 * (p.tile < 2 ? 512 : 256);
        break;
    }
    case LinearKernel::plain: break;
    }
    const bool fits = threads < 1ull << 32;
    out[0] = (unsigned long long)p.kernel;
    out[1] = (unsigned long long)p.tile;
    out[2] = grouped_fits(a.l.M, a.experts, a.l.N);
    out[3] = threads;
    out[4] = fits;
    if (p.kernel == LinearKernel::plain || (!fits && p.kernel != LinearKernel::tiled)) out[3] = (slots(16) * ((n + 15) / 16) + 3) / 4 * 256;
}

// Of rows, k, n, x_stride, group: {kernel, tile, whether such sizes are taken, threads of the launch}
extern "C" void ff_s4(const long long *size, int gated, int kernel, unsigned long long *out)
{
    LinearS4Args a = {};
    a.M = (int)size[0];
    a.K = (int)size[1];
    a.N = (int)size[2];
    a.ldx = size[3];
    a.group = (int)size[4];
    a.groups = (a.K + a.group - 1) / a.group;
    a.ldw = (a.K + 31) / 32 * 16;
    a.x = (const int8_t *)(1 << 24);
    a.w = (const uint8_t *)(2 << 24);
    a.w2 = gated ? (const uint8_t *)(3 << 24) : nullptr;
    const S4Plan p = plan_s4(a, LinearTuning{kernel, 0});
    const unsigned long long m = (unsigned long long)a.M, n = (unsigned long long)a.N;
    unsigned long long threads = 0;
    switch (p.kernel) {
    case LinearKernel::tokens: {
        const int k = a.K, along = k <= 2048 ? 1 : k <= 4096 ? 2 : k <= 8192 ? 4 : k <= 16384 ? 8 : 16, of = k > 16384 ? 4 : 8, waves = std::max(along, 4);
        const unsigned long long per = (unsigned long long)(gated ? of / 2 : of) * (waves / along);
        threads = (n + per - 1) / per * 64 * waves;
        break;
    }
    case LinearKernel::few: threads = (n + 15) / 16 * 512; break;
    case LinearKernel::tiled: {
        const int tile_m[] = {128, 128, 64, 32}, tile_n[] = {256, 128, gated ? 64 : 32, 32};
        const unsigned long long wide = (gated ? 2 : 1) * n;
        threads = ((m + tile_m[p.tile] - 1) / tile_m[p.tile] * ((wide + tile_n[p.tile] - 1) / tile_n[p.tile]) + 7) / 8 * 8 * 512;
        break;
    }
    case LinearKernel::plain: threads = ((m + 15) / 16 * ((n + 15) / 16) + 3) / 4 * 256;
    }
    out[0] = (unsigned long long)p.kernel;
    out[1] = (unsigned long long)p.tile;
    out[2] = s4_fits(a.M, a.N);
    out[3] = threads;
}

// An expert's positions as the kernels take them from any offsets
static void share_of(const int *offsets, int e, int positions, int *lo, int *hi)
{
    *lo = std::min(std::max(offsets[e], 0), positions);
    *hi = std::min(std::max(offsets[e + 1], *lo), positions);
}

template <Groups KIND>
static int groups_of(const int *offsets, int experts, int positions, int most)
{
    unsigned all = 0;                                      // (wraps around, as on the device)
    for (int e = 0; e < experts; ++e) {
        int lo, hi;
        share_of(offsets, e, positions, &lo, &hi);
        all += (unsigned)groups_among<kMixedRows, KIND>(hi - lo);
    }
    return std::min((int)all, most);
}

template <Groups KIND>
static bool place_of(const int *offsets, int experts, int positions, int slot, int *expert, int *m0, int *end)
{
    for (int e = 0; e < experts; ++e) {
        int lo, hi;
        share_of(offsets, e, positions, &lo, &hi);
        const int own = groups_among<kMixedRows, KIND>(hi - lo);
        if (slot < own) {
            *expert = e;
            *m0 = KIND >= kRest ? lo + (hi - lo) / kMixedRows * kMixedRows : lo + slot * kMixedRows;
            *end = hi;
            return slot >= 0;
        }
        slot -= own;
    }
    return false;
}

// The workgroups of a launch in tiles of several sizes, one after the other.  Rows in pieces of 64 from an expert's first one on, columns in pieces of 128:
// {pieces that no workgroup has, that several have, workgroups that lie outside, workgroups that have something}
template <bool EIGHTHS>
static void mixed(const int *offsets, int experts, int positions, int n, int steps, bool gated, long long *out)
{
    constexpr Groups REST = EIGHTHS ? kHalf : kRest;
    const int columns = gated ? 128 : 256, tiles_n = (n + columns - 1) / columns, tiles8_n = (n + 127) / 128, most = (int)grouped_slots(positions, experts, kMixedRows);
    const int groups = groups_of<kWholeOrMost>(offsets, experts, positions, most), rests = groups_of<REST>(offsets, experts, positions, most);
    const int small = EIGHTHS ? groups_of<kQuarter>(offsets, experts, positions, most) : 0;
    std::vector<long long> first(experts + 1, 0);          // an expert's first piece of rows
    for (int e = 0; e < experts; ++e) {
        int lo, hi;
        share_of(offsets, e, positions, &lo, &hi);
        first[e + 1] = first[e] + (hi - lo + 63) / 64;
    }
    std::vector<unsigned char> had((size_t)first[experts] * tiles8_n, 0);
    out[0] = out[1] = out[2] = out[3] = 0;
    const long long blocks = mixed_blocks<EIGHTHS>(positions, experts, tiles_n);
    for (long long b = 0; b < blocks; ++b) {
        const MixedTile t = mixed_tile<EIGHTHS>(groups, rests, small, tiles_n, tiles8_n, steps, (unsigned)b);
        if (t.rows == 0) continue;
        const int at = t.rows == 64 ? t.n : t.n * (columns / 128), wide = t.rows == 64 ? 1 : columns / 128;
        int e = 0, m0 = 0, end = 0;
        const bool some = t.from == kWholeOrMost ? place_of<kWholeOrMost>(offsets, experts, positions, t.slot, &e, &m0, &end)
                          : t.from == REST       ? place_of<REST>(offsets, experts, positions, t.slot, &e, &m0, &end)
                                                 : place_of<kQuarter>(offsets, experts, positions, t.slot, &e, &m0, &end);
        if (t.n < 0 || t.n >= (t.rows == 64 ? tiles8_n : tiles_n) || t.down < 0) {
            ++out[2];
            continue;
        }
        int lo, hi;
        share_of(offsets, e, positions, &lo, &hi);
        m0 += t.down;
        if (!some || m0 >= end) continue;
        ++out[3];
        if (m0 < lo || end > positions || (m0 - lo) % 64) {
            ++out[2];
            continue;
        }
        for (int r = (m0 - lo) / 64; r < (std::min(m0 + t.rows, end) - lo + 63) / 64; ++r)
            for (int c = at; c < std::min(at + wide, tiles8_n); ++c) {
                unsigned char &h = had[(size_t)(first[e] + r) * tiles8_n + c];
                h = (unsigned char)std::min(h + 1, 2);
            }
    }
    for (unsigned char h : had) {
        out[0] += h == 0;
        out[1] += h > 1;
    }
}

extern "C" void ff_mixed(const int *offsets, int experts, int positions, int n, int steps, int gated, int eighths, long long *out)
{
    if (eighths) mixed<true>(offsets, experts, positions, n, steps, gated, out);
    else mixed<false>(offsets, experts, positions, n, steps, gated, out);
}
