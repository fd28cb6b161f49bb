// How the kernels for products grouped by expert find their expert's positions.
#pragma once
#include "ffn_common.h"

namespace icnn {

// Positions m0 .. of expert `expert`, which has those up to `end`; expert -1: none
struct Place {
    int expert, m0, end;
};

// The experts' positions as a wave asks for them, all of its lanes together: lane l has the first 64 experts' l-th, so that a second question does not wait for memory again.
// The answers are the same in all lanes.  Whatever the offsets hold, the positions are in [0, M).
struct Shares {
    const GroupedArgs &g;
    int lo0, hi0;

    __device__ __forceinline__ explicit Shares(const GroupedArgs &args) : g(args) { load(0, &lo0, &hi0); }

    __device__ __forceinline__ void load(int base, int *lo, int *hi) const
    {
        const int e = base + (int)(threadIdx.x & 63), at = min(e, g.experts - 1), a = g.offsets[at], b = g.offsets[at + 1];
        *lo = min(max(a, 0), g.l.M);
        *hi = e < g.experts ? min(max(b, *lo), g.l.M) : *lo;
    }

    // How many groups there are
    template <int ROWS, Groups KIND>
    __device__ __forceinline__ int groups() const
    {
        int all = groups_among<ROWS, KIND>(hi0 - lo0);
        for (int base = 64; base < g.experts; base += 64) {
            int lo, hi;
            load(base, &lo, &hi);
            all += groups_among<ROWS, KIND>(hi - lo);
        }
        return __builtin_amdgcn_readlane(sums_up_to(all), 63);
    }

    // The `slot`-th of them, expert by expert
    template <int ROWS, Groups KIND = kAll>
    __device__ __forceinline__ Place place(int slot) const
    {
        Place p = {-1, 0, 0};
        int lo = lo0, hi = hi0;
        for (int base = 0;;) {
            const int own = groups_among<ROWS, KIND>(hi - lo);
            const int up = sums_up_to(own);
            const unsigned long long beyond = __ballot(up > slot);
            if (beyond) {
                const int at = __builtin_ctzll(beyond);
                const int before = __builtin_amdgcn_readlane(up - own, at), first = __builtin_amdgcn_readlane(lo, at);
                p.end = __builtin_amdgcn_readlane(hi, at);
                p.m0 = KIND >= kRest ? first + (p.end - first) / ROWS * ROWS : first + (slot - before) * ROWS;
                p.expert = p.m0 >= first && p.m0 < p.end ? base + at : -1;     // (always, but where sums of offsets that do not ascend have left 32 bits)
                return p;
            }
            slot -= __builtin_amdgcn_readlane(up, 63);
            base += 64;
            if (base >= g.experts) return p;
            load(base, &lo, &hi);
        }
    }
};

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
