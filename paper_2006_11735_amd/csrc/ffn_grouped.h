// How the kernels for products grouped by expert find their expert's positions.
#pragma once
#include "ffn_common.h"

namespace icnn {

// Positions m0 .. of expert `expert`, which has those up to `end`; expert -1: none
struct Place {
    int expert, m0, end;
};

// Groups of ROWS positions that there are
template <int ROWS>
__device__ __forceinline__ int groups_of(const GroupedArgs &g)
{
    int all = 0;
    for (int e = threadIdx.x & 63; e < g.experts; e += 64) {
        const int lo = min(max(g.offsets[e], 0), g.l.M), hi = min(max(g.offsets[e + 1], lo), g.l.M);
        all += (hi - lo + ROWS - 1) / ROWS;
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d);
    return __builtin_amdgcn_readfirstlane(all);
}

// The `slot`-th group of ROWS positions (the last one of an expert may have fewer), expert by expert.  A wave asks, all of its lanes together; the answer is the same in
// all.  Whatever the offsets hold, the positions returned are in [0, M).
template <int ROWS>
__device__ __forceinline__ Place place_of(const GroupedArgs &g, int slot)
{
    const int lane = threadIdx.x & 63;
    Place p = {-1, 0, 0};
    for (int base = 0; base < g.experts; base += 64) {
        const int e = min(base + lane, g.experts - 1);
        const int lo = min(max(g.offsets[e], 0), g.l.M), hi = min(max(g.offsets[e + 1], lo), g.l.M);
        const int own = base + lane < g.experts ? (hi - lo + ROWS - 1) / ROWS : 0;
        int up = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int below = __shfl_up(up, d);
            if (lane >= d) up += below;
        }
        const unsigned long long beyond = __ballot(up > slot);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            const int before = __builtin_amdgcn_readlane(up - own, at);
            const int first = __builtin_amdgcn_readlane(lo, at);
            p.m0 = first + (slot - before) * ROWS;
            p.end = __builtin_amdgcn_readlane(hi, at);
            p.expert = p.m0 >= first && p.m0 < p.end ? base + at : -1;         // (always, but where sums of offsets that do not ascend have left 32 bits)
            return p;
        }
        slot -= __builtin_amdgcn_readlane(up, 63);
    }
    return p;
}

// x's row of position m: -1 where the index names none
__device__ __forceinline__ int row_of(const GroupedArgs &g, int m)
{
    if (!g.index) return m;
    const int r = g.index[m];
    return r >= 0 && r < g.x_rows ? r : -1;
}

// The operands of expert e's product, whose positions end at `end`
template <bool GATED>
__device__ __forceinline__ LinearArgs of_expert(const GroupedArgs &g, int e, int end)
{
    LinearArgs a = g.l;
    a.M = end;
    const long long first = (long long)e * a.N;
    a.w += e * g.expert_stride;
    a.ws += first;
    if (a.bias) a.bias += first;
    if (GATED) {
        a.w2 += e * g.expert_stride;
        a.ws2 += first;
        if (a.bias2) a.bias2 += first;
    }
    return a;
}

}  // namespace icnn
