// The router of a layer of experts: a token's `top` largest logits, their gates, and all tokens' choices in the order of the experts.
//   softmax: g_j = scale exp(l_j - max) / sum of exp(l - max), over all of the row or, normalised, over the chosen;  sigmoid: g_j = scale / (1 + exp(-l_j)), or that
//   over the chosen ones' sum.  place: a stable counting sort by expert, so a choice's position is the number of choices of lower experts and of its expert's by
//   earlier tokens: counts and bit masks, whose order of arrival changes nothing.
// What bounds it is latency: a launch, or two with what is between them.
#include "ffn_common.h"

#include <type_traits>

namespace icnn {

namespace {

// Tokens that share one mask of 32 bits an expert; chunks of so many masks a workgroup, counted in 16 bits
constexpr int kMask = 32, kWantedChunks = 256, kMostChunk = 32768;

long long chunk_of(long long rows)
{
    const long long per = ((rows + kWantedChunks - 1) / kWantedChunks + kMask - 1) / kMask * kMask;
    return per < kMostChunk ? per : kMostChunk;
}

// Logits as numbers that are ordered as they are: 0 for what is never chosen (minus infinity, places behind the last expert), all ones for a NaN
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);          // (minus zero is zero)
    const uint32_t key = b ^ (b >> 31 ? ~0u : 0x80000000u);
    return v != v ? ~0u : v == -__builtin_huge_valf() ? 0 : key;
}

__device__ __forceinline__ float value_of_key(uint32_t key)
{
    if (key == ~0u) return __builtin_nanf("");
    return __builtin_bit_cast(float, key ^ (key >> 31 ? 0x80000000u : ~0u));
}

template <int LANES, class F>
__device__ __forceinline__ auto over_lanes(decltype(F{}(0, 0)) v, F f)
{
#pragma unroll
    for (int d = LANES / 2; d; d >>= 1) v = f(v, __shfl_xor(v, d));
    return v;
}

struct MaxU {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct SumF {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// Exclusive sums of `experts` counts in LDS, by all threads of the workgroup; the total is returned
template <int THREADS>
__device__ __forceinline__ int scan_counts(int *counts, int *first, int experts)
{
    constexpr int PER = kMostExperts / THREADS < 1 ? 1 : kMostExperts / THREADS, WAVES = THREADS / 64;
    __shared__ int sums[WAVES];
    const int t = threadIdx.x, lane = t & 63;
    int mine[PER], own = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        mine[i] = t * PER + i < experts ? counts[t * PER + i] : 0;
        own += mine[i];
    }
    int up = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int below = __shfl_up(up, d);
        if (lane >= d) up += below;
    }
    if (lane == 63) sums[t >> 6] = up;
    __syncthreads();
    int before = up - own, total = 0;
#pragma unroll
    for (int q = 0; q < WAVES; ++q) {
        if (q < t >> 6) before += sums[q];
        total += sums[q];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (t * PER + i < experts) first[t * PER + i] = before;
        before += mine[i];
    }
    __syncthreads();
    return total;
}

}  // namespace

// LANES lanes a token with P experts each, next to each other: among equal ones the lowest lane's first has the lowest index.  ONE: all rows are this workgroup's, which
// then places them too.
template <int LANES, int P, bool ONE>
__global__ __launch_bounds__(256) void route_choose_kernel(const RouteArgs a, int chunk)
{
    constexpr int TOKENS = 256 / LANES;                    // at a time
    __shared__ uint32_t mask[kMostExperts];
    __shared__ int counts[kMostExperts], first[ONE ? kMostExperts : 1];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const long long begin = (long long)blockIdx.x * chunk;
    const int mine = (int)min((long long)chunk, a.rows - begin);
    const unsigned long long own_lanes = (LANES == 64 ? ~0ull : (1ull << LANES) - 1) << (threadIdx.x & 63) / LANES * LANES;
    for (int e = threadIdx.x; e < a.experts; e += 256) {
        mask[e] = 0;
        counts[e] = 0;
    }
    __syncthreads();
    for (int base = 0; base < mine; base += kMask) {
#pragma unroll 1
        for (int at = base; at < min(base + kMask, mine); at += TOKENS) {
            const bool some = at + slot < min(base + kMask, mine);
            const long long t = begin + at + (some ? slot : 0);
            uint32_t key[P], best = 0;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int e = lane * P + i;
                const float v = load_number(a.logits, t * a.ld + min(e, a.experts - 1), a.dtype);
                key[i] = e < a.experts ? key_of(v) : 0;
                best = max(best, key[i]);
            }
            const uint32_t largest = over_lanes<LANES>(best, MaxU{});
            const float most = value_of_key(largest);
            float every = 0.f;
            if (a.score == 0 && !a.normalise) {
#pragma unroll
                for (int i = 0; i < P; ++i) every += key[i] ? expf(value_of_key(key[i]) - most) : 0.f;
                every = over_lanes<LANES>(every, SumF{});
            }
            uint32_t chosen = 0;                           // lane j has the token's choice j
            int which = -1;
            for (int j = 0; j < a.top; ++j) {
                const uint32_t m = over_lanes<LANES>(best, MaxU{});
                const unsigned long long has = __ballot(best == m && m != 0) & own_lanes;
                const int winner = has ? __builtin_ctzll(has) : -1;
                int hit = -1;
                uint32_t next = 0;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const bool takes = winner == (int)(threadIdx.x & 63) && hit < 0 && key[i] == m;
                    hit = takes ? i : hit;
                    key[i] = takes ? 0 : key[i];
                    next = max(next, key[i]);
                }
                best = next;
                const int e = __shfl(lane * P + hit, winner < 0 ? 0 : winner);
                if (lane == j && winner >= 0) {
                    chosen = m;
                    which = e;
                }
            }
            const float l = value_of_key(chosen);
            float g;
            if (a.score == 0) {
                g = which >= 0 ? expf(l - most) : 0.f;
            } else {
                // exp(l) / (1 + exp(l)), where it is to be normalised over the largest one's exp if that is below 1: sums of what has left float32 would be 0
                const float shift = a.normalise && most < 0.f ? most : 0.f;
                g = which < 0 ? 0.f : l > 0.f ? 1.f / (1.f + expf(-l)) : expf(l - shift) / (1.f + expf(l));
            }
            const float sum = a.normalise ? over_lanes<LANES>(g, SumF{}) : a.score == 0 ? every : 1.f;
            if (some && lane < a.top) {
                a.expert[t * a.top + lane] = which;
                a.gate[t * a.top + lane] = which >= 0 ? g / sum * a.scale : 0.f;
                if (which >= 0) atomicOr(&mask[which], 1u << (at - base + slot));
            }
        }
        if (!ONE) {
            __syncthreads();
            for (int e = threadIdx.x; e < a.experts; e += 256) {
                counts[e] += __popc(mask[e]);
                mask[e] = 0;
            }
            __syncthreads();
        }
    }
    if (ONE) {                                             // (one mask an expert holds all rows)
        __syncthreads();
        for (int e = threadIdx.x; e < a.experts; e += 256) counts[e] = __popc(mask[e]);
        __syncthreads();
        const int total = scan_counts<256>(counts, first, a.experts);
        for (int e = threadIdx.x; e < a.experts; e += 256) a.offsets[e] = first[e];
        if (threadIdx.x == 0) a.offsets[a.experts] = total;
        for (int i = total + threadIdx.x; i < mine * a.top; i += 256) a.token[i] = -1;
        for (int i = threadIdx.x; i < mine * a.top; i += 256) {
            const int t = i / a.top, e = a.expert[i];      // (this workgroup's own, written in front of a barrier)
            int p = -1;
            if (e >= 0) {
                p = first[e] + __popc(mask[e] & ((1u << t) - 1));
                a.token[p] = t;
            }
            a.place[i] = p;
        }
    } else {
        for (int e = threadIdx.x; e < a.experts; e += 256) a.counts[(long long)blockIdx.x * a.experts + e] = (uint16_t)counts[e];
    }
}

// The places of a chunk's choices, from all chunks' counts.
__global__ __launch_bounds__(1024) void route_place_kernel(const RouteArgs a, int chunk)
{
    __shared__ uint32_t mask[kMostExperts];
    __shared__ int total[kMostExperts], before[kMostExperts], first[kMostExperts];
    const int chunks = gridDim.x, t = threadIdx.x;
    const long long begin = (long long)blockIdx.x * chunk;
    const int mine = (int)min((long long)chunk, a.rows - begin);
    for (int e = t; e < a.experts; e += 1024) {
        mask[e] = 0;
        total[e] = before[e] = 0;
    }
    __syncthreads();
    // 1024 / experts threads an expert, each every so many-th chunk
    const int ways = 1024 / a.experts, e0 = t % a.experts, way = t / a.experts;
    if (way < ways) {
        int all = 0, low = 0;
        for (int q = way; q < chunks; q += ways) {
            const int v = a.counts[(long long)q * a.experts + e0];
            all += v;
            low += q < (int)blockIdx.x ? v : 0;
        }
        atomicAdd(&total[e0], all);
        atomicAdd(&before[e0], low);
    }
    __syncthreads();
    const int sum = scan_counts<1024>(total, first, a.experts);
    if (blockIdx.x == 0) {
        for (int e = t; e < a.experts; e += 1024) a.offsets[e] = first[e];
        if (t == 0) a.offsets[a.experts] = sum;
    }
    for (long long i = sum + (long long)blockIdx.x * 1024 + t; i < a.rows * a.top; i += (long long)chunks * 1024) a.token[i] = -1;
    if (t < a.experts) first[t] += before[t];
    __syncthreads();
    for (int base = 0; base < mine; base += kMask) {
        const int many = min(kMask, mine - base) * a.top;  // (at most 512)
        const long long at = (begin + base) * a.top;
        const int e = t < many ? a.expert[at + t] : -1, row = t / a.top;
        if (e >= 0) atomicOr(&mask[e], 1u << row);
        __syncthreads();
        if (t < many) {
            int p = -1;
            if (e >= 0) {
                p = first[e] + __popc(mask[e] & ((1u << row) - 1));
                a.token[p] = (int)(begin + base + row);
            }
            a.place[at + t] = p;
        }
        __syncthreads();
        if (t < a.experts) {
            first[t] += __popc(mask[t]);
            mask[t] = 0;
        }
        __syncthreads();
    }
}

size_t route_workspace(long long rows, int experts)
{
    if (rows <= kMask) return 0;
    const long long chunk = chunk_of(rows);
    return (size_t)((rows + chunk - 1) / chunk) * (size_t)experts * 2;
}

template <int LANES, int P>
static hipError_t launch_choose(const RouteArgs &a, hipStream_t st)
{
    if (a.rows <= kMask) {
        hipLaunchKernelGGL((route_choose_kernel<LANES, P, true>), dim3(1), dim3(256), 0, st, a, kMask);
        return hipGetLastError();
    }
    const long long chunk = chunk_of(a.rows);
    const unsigned chunks = (unsigned)((a.rows + chunk - 1) / chunk);
    hipLaunchKernelGGL((route_choose_kernel<LANES, P, false>), dim3(chunks), dim3(256), 0, st, a, (int)chunk);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL(route_place_kernel, dim3(chunks), dim3(1024), 0, st, a, (int)chunk);
    return hipGetLastError();
}

hipError_t launch_route(const RouteArgs &a, hipStream_t st)
{
    if (a.experts <= 16) return launch_choose<16, 1>(a, st);
    if (a.experts <= 64) return launch_choose<16, 4>(a, st);
    if (a.experts <= 128) return launch_choose<16, 8>(a, st);
    if (a.experts <= 256) return launch_choose<16, 16>(a, st);
    if (a.experts <= 512) return launch_choose<32, 16>(a, st);
    return launch_choose<64, 16>(a, st);
}

}  // namespace icnn
