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
