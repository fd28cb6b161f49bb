// The planning of products of 8-bit rows (csrc/ffn_plan.h), by itself, for tests without a GPU.
#include "../paper_2006_11735_amd/csrc/ffn_plan.h"

using namespace icnn;

static LinearArgs args_of(const long long *size, bool gated, uintptr_t x, uintptr_t w, uintptr_t w2)
{
    LinearArgs a = {};
    a.M = (int)size[0];
    a.K = (int)size[1];
    a.N = (int)size[2];
    a.ldx = size[3];
    a.ldw = size[4];
    a.x = (const int8_t *)x;
    a.w = (const int8_t *)w;
    a.w2 = gated ? (const int8_t *)w2 : nullptr;
    return a;
}

// The launches of a product: how many, and of the one with most threads its threads (at most) and its kernel
extern "C" void ff_launches(const long long *size, int gated, int kernel, unsigned long long *out)
{
    const LinearArgs whole = args_of(size, gated, 1 << 24, 2 << 24, 3 << 24);
    const LinearTuning tuning = {kernel, 0};
    out[0] = out[1] = out[2] = 0;
    const unsigned long long tile_threads[] = {512, 512, 256, 256, 256, 256};
    each_range(whole, 2, [&](const LinearArgs &a) {
        const LinearPlan p = plan_launch(a, tuning);
        const unsigned long long m = (unsigned long long)a.M, n = (unsigned long long)a.N * (gated ? 2 : 1), one = (unsigned long long)a.N;
        unsigned long long threads = 0;
        switch (p.kernel) {
        case LinearKernel::tokens: threads = one * (gated ? 512 : 256); break;
        case LinearKernel::few: threads = (one + 15) / 16 * 256; break;
        case LinearKernel::tiled: {
            const TileCost &t = kTiles[p.tiles.tile];
            threads = ((m + t.m - 1) / t.m * ((n + t.n - 1) / t.n) + 7) * tile_threads[p.tiles.tile];
            break;
        }
        case LinearKernel::plain: threads = ((m + 15) / 16 * ((one + 15) / 16) + 3) / 4 * 256;
        }
        ++out[0];
        if (threads >= out[1]) {
            out[1] = threads;
            out[2] = (unsigned long long)p.kernel;
        }
        return 0;
    });
}

// The ranges of rows and outputs that a product goes in: {first row, rows, first output, outputs} each, at most `most` of them; every operand's place is checked
extern "C" int ff_ranges(const long long *size, int gated, int most, long long *out)
{
    LinearArgs whole = args_of(size, gated, 1 << 24, 2 << 24, 3 << 24);
    int8_t *const far = (int8_t *)(1ull << 50);
    whole.ldr = size[2] + 3;
    whole.ldy = size[2] + 5;
    whole.xs = (const float *)far;
    whole.ws = (const float *)(2 * (uintptr_t)far);
    whole.ws2 = gated ? (const float *)(3 * (uintptr_t)far) : nullptr;
    whole.bias = (const float *)(4 * (uintptr_t)far);
    whole.bias2 = nullptr;
    whole.res = gated ? nullptr : (const void *)(5 * (uintptr_t)far);
    whole.y = (void *)(6 * (uintptr_t)far);
    whole.workspace = (void *)16;
    int n = 0;
    return each_range(whole, 2, [&](const LinearArgs &a) {
        if (n == most) return 1;
        const long long m0 = (a.x - whole.x) / whole.ldx, n0 = (a.w - whole.w) / whole.ldw;
        const bool good = a.x == whole.x + m0 * whole.ldx && a.w == whole.w + n0 * whole.ldw && a.xs == whole.xs + m0 && a.ws == whole.ws + n0 &&
                          a.bias == whole.bias + n0 && !a.bias2 && (gated ? a.w2 == whole.w2 + n0 * whole.ldw && a.ws2 == whole.ws2 + n0 && !a.res
                                                                         : !a.w2 && !a.ws2 && a.res == (const int8_t *)whole.res + (m0 * whole.ldr + n0) * 2) &&
                          a.y == (int8_t *)whole.y + (m0 * whole.ldy + n0) * 2 && (a.workspace == nullptr || (a.M == whole.M && a.N == whole.N));
        if (!good) return 2;
        out[4 * n] = m0;
        out[4 * n + 1] = a.M;
        out[4 * n + 2] = n0;
        out[4 * n + 3] = a.N;
        ++n;
        return 0;
    }) ? -1 : n;
}

// Of rows, k, n, x_stride, w_stride and the addresses of x, w and w_up: {kernel, tile, ranges of k, bytes of the workspace} of a launch with or without a workspace
extern "C" void ff_launch(const long long *size, int gated, uintptr_t x, uintptr_t w, uintptr_t w2, int with_workspace, int kernel, int split, unsigned long long *out)
{
    LinearArgs a = args_of(size, gated, x, w, w2);
    a.workspace = with_workspace ? (void *)16 : nullptr;
    const LinearPlan p = plan_launch(a, LinearTuning{kernel, split});
    out[0] = (unsigned long long)p.kernel;
    out[1] = (unsigned long long)p.tiles.tile;
    out[2] = (unsigned long long)p.tiles.splits;
    out[3] = plan_workspace(a, p);
}
