// The router of a layer of experts: a token's `top` largest logits, their gates, and all tokens' choices in the order of the experts.
//   softmax: g_j = scale exp(l_j - max) / sum of exp(l - max), over all of the row or, normalised, over the chosen;  sigmoid: g_j = scale / (1 + exp(-l_j)), or that
//   over the chosen ones' sum.  place: a stable counting sort by expert, so a choice's position is the number of choices of lower experts and of its expert's by
//   earlier tokens: counts and bit masks, whose order of arrival changes nothing.
// What bounds it is latency: a launch, or two with what is between them.
#include "ffn_common.h"

#include <type_traits>

namespace icnn {

namespace {

// Tokens that share one mask of 32 bits an expert; chunks of whole masks a workgroup, counted in 8 bits or 16
constexpr int kMask = 32, kWantedChunks = 256, kMostChunk = 32768;

long long chunk_of(long long rows)
{
    const long long per = ((rows + kWantedChunks - 1) / kWantedChunks + kMask - 1) / kMask * kMask;
    return per < kMostChunk ? per : kMostChunk;
}

int count_bytes(long long chunk) { return chunk < 256 ? 1 : 2; }

// Logits as numbers that are ordered as they are, of which 0 is never chosen (minus infinity, places behind the last expert).  A 16-bit logit leaves room for its expert,
// counted from above: the numbers of a row are all different then, and the largest of equal logits is the lowest expert's.
template <int DT>
__device__ __forceinline__ uint32_t key_of(uint32_t bits, int e)
{
    const float v = value_of(bits, DT);
    if (v == -__builtin_huge_valf()) return 0;
    if constexpr (DT == kF32) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);      // (minus zero is zero)
        return v != v ? ~0u : b ^ (b >> 31 ? ~0u : 0x80000000u);
    } else {
        const uint32_t b = v == 0.f ? 0 : bits, key = v != v ? 0xffffu : b ^ (b >> 15 ? 0xffffu : 0x8000u);
        return key << 16 | (0xffffu - (uint32_t)e);
    }
}

template <int DT>
__device__ __forceinline__ float value_of_key(uint32_t key)
{
    if constexpr (DT == kF32) {
        return key == ~0u ? __builtin_nanf("") : __builtin_bit_cast(float, key ^ (key >> 31 ? 0x80000000u : ~0u));
    } else {
        const uint32_t k = key >> 16;
        return k == 0xffffu ? __builtin_nanf("") : value_of(k ^ (k >> 15 ? 0x8000u : 0xffffu), DT);
    }
}

// f over LANES lanes next to each other, in all of them
template <int LANES, class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f)
{
    static_assert(LANES >= 16 && LANES <= 64, "rows of sixteen lanes");
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));          // lanes ^ 1
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));          // lanes ^ 2
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));         // eight lanes mirrored
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));         // sixteen lanes mirrored
    if (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = f(r[0], r[1]);
    }
    if (LANES == 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = f(r[0], r[1]);
    }
    return v;
}

struct Largest {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct Least {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a < b ? a : b; }
};
struct Sum {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b)); }
};

template <int LANES>
__device__ __forceinline__ float sum_over(float v)
{
    return __builtin_bit_cast(float, over_lanes<LANES>(__builtin_bit_cast(uint32_t, v), Sum{}));
}

// The sum over a wave's lanes that are a multiple of `side` (1, 2 or 4) apart, in all of them
__device__ __forceinline__ int sum_apart(int v, int side)
{
    const auto r = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
    v = (int)(r[0] + r[1]);
    const auto q = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
    v = (int)(q[0] + q[1]);
    v += __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true);         // sixteen lanes turned by 8, by 4, ...
    v += __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, true);
    if (side <= 2) v += __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, true);
    if (side == 1) v += __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, true);
    return v;
}

// first[e] = the sum of count(0 .. e - 1), by all threads of the workgroup; the total is returned
template <int THREADS, class F>
__device__ __forceinline__ int scan_counts(int experts, int *first, F &&count)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ int sums[WAVES];
    const int t = threadIdx.x, lane = t & 63;
    int total = 0;
    for (int base = 0; base < experts; base += THREADS) {
        const int own = base + t < experts ? count(base + t) : 0;
        const int up = sums_up_to(own);
        if (WAVES > 1) {
            if (base) __syncthreads();                     // (the sums of the turn before have been read)
            if (lane == 63) sums[t >> 6] = up;
            __syncthreads();
        }
        int before = total + up - own;
        if (WAVES > 1) {
#pragma unroll
            for (int q = 0; q < WAVES; ++q) {
                if (q < t >> 6) before += sums[q];
                total += sums[q];
            }
        } else {
            total += __builtin_amdgcn_readlane(up, 63);
        }
        if (base + t < experts) first[base + t] = before;
    }
    return total;
}

}  // namespace

// LANES lanes a token with P experts each, next to each other.  ONE: all rows are this workgroup's, which then places them too.
// As many threads as a mask's tokens want, at most 1024: by half of them, in two turns, 8192 x 256, top 8 took 8.6 us instead of 6.2; one wave for a few tokens
template <int LANES>
constexpr int kChooseThreads = kMask * LANES < 1024 ? kMask * LANES : 1024;

template <int LANES, int P, int DT, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void route_choose_kernel(const RouteArgs a, int chunk)
{
    constexpr int TOKENS = THREADS / LANES;                // at a time
    __shared__ uint32_t mask[kMostExperts];
    __shared__ int counts[kMostExperts], first[ONE ? kMostExperts : 1];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES, e0 = lane * P;
    const long long begin = (long long)blockIdx.x * chunk;
    const int mine = (int)min((long long)chunk, a.rows - begin);
    for (int e = threadIdx.x; e < a.experts; e += THREADS) {
        mask[e] = 0;
        counts[e] = 0;
    }
    __syncthreads();
    for (int base = 0; base < mine; base += kMask) {
#pragma unroll 1
        for (int at = base; at < min(base + kMask, mine); at += TOKENS) {
            const bool some = at + slot < min(base + kMask, mine);
            const long long t = begin + at + (some ? slot : 0);
            uint32_t key[P], bits[P], best = 0;
            if (P % 8 == 0 && a.experts == LANES * P) {
#pragma unroll
                for (int i = 0; i < P / 8; ++i) {
                    const Eight<DT> v = load_eight<DT>(a.logits, t * a.ld + e0 + 8 * i);
#pragma unroll
                    for (int q = 0; q < 8; ++q) bits[(8 * i + q) % P] = DT == kF32 ? (uint32_t)v.b[DT == kF32 ? q >> 2 : 0][q & 3] : (uint32_t)v.b[0][q >> 1] >> (16 * (q & 1)) & 0xffffu;
                }
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i) bits[i] = load_bits(a.logits, t * a.ld + min(e0 + i, a.experts - 1), DT);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                key[i] = e0 + i < a.experts ? key_of<DT>(bits[i], e0 + i) : 0;
                best = max(best, key[i]);
            }
            const uint32_t largest = over_lanes<LANES>(best, Largest{});
            const float most = value_of_key<DT>(largest);
            float every = 0.f;
            if (a.score == 0 && !a.normalise) {
#pragma unroll
                for (int i = 0; i < P; ++i) every += key[i] ? expf(value_of_key<DT>(key[i]) - most) : 0.f;
                every = sum_over<LANES>(every);
            }
            uint32_t chosen = 0, m = largest;              // lane j has the token's choice j
            int which = -1;
            for (int j = 0; j < a.top; ++j) {
                uint32_t e;
                if constexpr (DT == kF32) {                // the lowest of those that have it
                    uint32_t lowest = ~0u;
#pragma unroll
                    for (int i = P - 1; i >= 0; --i) lowest = key[i] == m ? e0 + i : lowest;
                    e = over_lanes<LANES>(lowest, Least{});
                } else {
                    e = 0xffffu - (m & 0xffffu);
                }
                if (lane == j && m) {
                    chosen = m;
                    which = (int)e;
                }
                best = 0;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    key[i] = (DT == kF32 ? e == (uint32_t)(e0 + i) : key[i] == m) ? 0 : key[i];
                    best = max(best, key[i]);
                }
                m = over_lanes<LANES>(best, Largest{});
            }
            const float l = value_of_key<DT>(chosen);
            float g;
            if (a.score == 0) {
                g = which >= 0 ? expf(l - most) : 0.f;
            } else {
                // exp(l) / (1 + exp(l)), where it is to be normalised over the largest one's exp if that is below 1: sums of what has left float32 would be 0
                const float shift = a.normalise && most < 0.f ? most : 0.f;
                g = which < 0 ? 0.f : l > 0.f ? 1.f / (1.f + expf(-l)) : expf(l - shift) / (1.f + expf(l));
            }
            const float sum = a.normalise ? sum_over<LANES>(g) : a.score == 0 ? every : 1.f;
            if (some && lane < a.top) {
                a.expert[t * a.top + lane] = which;
                a.gate[t * a.top + lane] = which >= 0 ? g / sum * a.scale : 0.f;
                if (which >= 0) atomicOr(&mask[which], 1u << (at - base + slot));
            }
        }
        if (!ONE) {
            __syncthreads();
            for (int e = threadIdx.x; e < a.experts; e += THREADS) {
                counts[e] += __popc(mask[e]);
                mask[e] = 0;
            }
            __syncthreads();
        }
    }
    if (ONE) {                                             // (one mask an expert holds all rows)
        __syncthreads();
        const int total = scan_counts<THREADS>(a.experts, first, [&](int e) { return __popc(mask[e]); });
        __syncthreads();
        for (int e = threadIdx.x; e < a.experts; e += THREADS) a.offsets[e] = first[e];
        if (threadIdx.x == 0) a.offsets[a.experts] = total;
        for (int i = total + threadIdx.x; i < mine * a.top; i += THREADS) a.token[i] = -1;
        for (int i = threadIdx.x; i < mine * a.top; i += THREADS) {
            const int t = i / a.top, e = a.expert[i];      // (this workgroup's own, written in front of a barrier)
            int p = -1;
            if (e >= 0) {
                p = first[e] + __popc(mask[e] & ((1u << t) - 1));
                a.token[p] = t;
            }
            a.place[i] = p;
        }
    } else {
        for (int e = threadIdx.x; e < a.experts; e += THREADS) {
            if (chunk < 256) ((uint8_t *)a.counts)[(long long)blockIdx.x * ((a.experts + 15) / 16 * 16) + e] = (uint8_t)counts[e];
            else ((uint16_t *)a.counts)[(long long)blockIdx.x * ((a.experts + 7) / 8 * 8) + e] = (uint16_t)counts[e];
        }
    }
}

// The places of a chunk's choices, from all chunks' counts, of BYTES each.
constexpr int kPlaceThreads = 512;

template <int BYTES, bool FOLD>
__global__ __launch_bounds__(kPlaceThreads) void route_place_kernel(const RouteArgs a, int chunk)
{
    constexpr int THREADS = kPlaceThreads, EACH = 16 / BYTES, CHOICES = kMask * kMostTop / THREADS;
    __shared__ uint32_t mask[kMostExperts];
    __shared__ int total[kMostExperts], before[kMostExperts], first[kMostExperts];         // expert EACH p + e's at e * pieces + p: lanes that add meet no bank twice
    const int chunks = gridDim.x, t = threadIdx.x;
    const long long begin = (long long)blockIdx.x * chunk;
    const int mine = (int)min((long long)chunk, a.rows - begin), pieces = (a.experts + EACH - 1) / EACH;
    auto slot_of = [&](int e) { return e % EACH * pieces + e / EACH; };
    // (a mask's choices, on their way early)
    int chosen[CHOICES];
    auto fetch = [&](int base) {
#pragma unroll
        for (int i = 0; i < CHOICES; ++i) {
            const int c = i * THREADS + t;
            chosen[i] = c < min(kMask, mine - base) * a.top ? a.expert[(begin + base) * a.top + c] : -1;
        }
    };
    fetch(0);
    for (int e = t; e < kMostExperts; e += THREADS) mask[e] = total[e] = before[e] = 0;
    __syncthreads();
    // A thread has 16 bytes of counts of every so many-th chunk
    // (FOLD, up to four pieces: lanes of one piece are `side` apart, a power of two, and add up before they all go to the same words of LDS; 8192 x 8 20 us without, 8.6
    // with, 8192 x 256 11.9 and 14.3)
    const int side = !FOLD ? pieces : pieces == 3 ? 4 : pieces;
    const int ways = THREADS / side, piece = t % side, way = t / side;
    if (t / 64 * 64 < chunks * side) {                     // (waves that have a chunk)
        int all[EACH] = {}, low[EACH] = {};
        // (bytes are added two to a register, 16 bits each: no more than 256 chunks of less than 256 rows have counts of a byte)
        uint32_t all2[8] = {}, low2[8] = {};
#pragma unroll 4
        for (int q = way; q < chunks; q += ways) {
            const v4i v = *((const v4i *)a.counts + (long long)q * pieces + (FOLD ? min(piece, pieces - 1) : piece));
            const uint32_t lower = q < (int)blockIdx.x ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (BYTES == 1) {
                    const uint32_t even = (uint32_t)v[i] & 0xff00ffu, odd = (uint32_t)v[i] >> 8 & 0xff00ffu;
                    all2[2 * i] += even;
                    all2[2 * i + 1] += odd;
                    low2[2 * i] += even & lower;
                    low2[2 * i + 1] += odd & lower;
                } else {
                    const int n0 = v[i] & 0xffff, n1 = (int)((uint32_t)v[i] >> 16);
                    all[2 * i] += n0;
                    all[2 * i + 1] += n1;
                    low[2 * i] += n0 & (int)lower;
                    low[2 * i + 1] += n1 & (int)lower;
                }
            }
        }
        if constexpr (FOLD) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (BYTES == 1) {
                    all2[i] = sum_apart((int)all2[i], side);
                    low2[i] = sum_apart((int)low2[i], side);
                } else {
                    all[i] = sum_apart(all[i], side);
                    low[i] = sum_apart(low[i], side);
                }
            }
        }
        if constexpr (BYTES == 1) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                all[e] = (int)(all2[(e >> 2) * 2 + (e & 1)] >> (8 * (e & 2)) & 0xffffu);
                low[e] = (int)(low2[(e >> 2) * 2 + (e & 1)] >> (8 * (e & 2)) & 0xffffu);
            }
        }
        if (FOLD ? (t & 63) < pieces : way < min(ways, chunks)) {
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (EACH * piece + e < a.experts) {
                    atomicAdd(&total[e * pieces + piece], all[e]);
                    atomicAdd(&before[e * pieces + piece], low[e]);
                }
        }
    }
    __syncthreads();
    // first[e]: the places of lower experts, and of this one's in front of the chunk
    const int sum = scan_counts<THREADS>(a.experts, first, [&](int e) { return total[slot_of(e)]; });
    for (int e = t; e < a.experts; e += THREADS) {         // (each thread its own)
        if (blockIdx.x == 0) a.offsets[e] = first[e];
        first[e] += before[slot_of(e)];
    }
    if (blockIdx.x == 0 && t == 0) a.offsets[a.experts] = sum;
    for (long long i = sum + (long long)blockIdx.x * THREADS + t; i < a.rows * a.top; i += (long long)chunks * THREADS) a.token[i] = -1;
    for (int base = 0; base < mine; base += kMask) {
        const int many = min(kMask, mine - base) * a.top;
        const long long at = (begin + base) * a.top;
        if (base) fetch(base);
#pragma unroll
        for (int i = 0; i < CHOICES; ++i)
            if (chosen[i] >= 0) atomicOr(&mask[chosen[i]], 1u << ((i * THREADS + t) / a.top));
        __syncthreads();
#pragma unroll
        for (int i = 0; i < CHOICES; ++i) {
            const int c = i * THREADS + t, row = c / a.top;
            if (c >= many) continue;
            int p = -1;
            if (chosen[i] >= 0) {
                p = first[chosen[i]] + __popc(mask[chosen[i]] & ((1u << row) - 1));
                a.token[p] = (int)(begin + base + row);
            }
            a.place[at + c] = p;
        }
        if (base + kMask < mine) {
            __syncthreads();
            for (int e = t; e < a.experts; e += THREADS) {
                first[e] += __popc(mask[e]);
                mask[e] = 0;
            }
            __syncthreads();
        }
    }
}

size_t route_workspace(long long rows, int experts)
{
    if (rows <= kMask) return 0;
    const long long chunk = chunk_of(rows);
    return (size_t)((rows + chunk - 1) / chunk) * (size_t)((experts * count_bytes(chunk) + 15) / 16) * 16;
}

template <int LANES, int P, int DT>
static hipError_t launch_of(const RouteArgs &a, hipStream_t st)
{
    constexpr int MANY = kChooseThreads<LANES>;
    if (a.rows <= 64 / LANES) {
        hipLaunchKernelGGL((route_choose_kernel<LANES, P, DT, 64, true>), dim3(1), dim3(64), 0, st, a, kMask);
        return hipGetLastError();
    }
    if (a.rows <= kMask) {
        hipLaunchKernelGGL((route_choose_kernel<LANES, P, DT, MANY, true>), dim3(1), dim3(MANY), 0, st, a, kMask);
        return hipGetLastError();
    }
    const long long chunk = chunk_of(a.rows);
    const unsigned chunks = (unsigned)((a.rows + chunk - 1) / chunk);
    hipLaunchKernelGGL((route_choose_kernel<LANES, P, DT, MANY, false>), dim3(chunks), dim3(MANY), 0, st, a, (int)chunk);
    if (hipError_t e = hipGetLastError()) return e;
    const int bytes = count_bytes(chunk);
    const bool fold = (a.experts * bytes + 15) / 16 <= 4;
    if (bytes == 1 && fold) hipLaunchKernelGGL((route_place_kernel<1, true>), dim3(chunks), dim3(kPlaceThreads), 0, st, a, (int)chunk);
    else if (bytes == 1) hipLaunchKernelGGL((route_place_kernel<1, false>), dim3(chunks), dim3(kPlaceThreads), 0, st, a, (int)chunk);
    else if (fold) hipLaunchKernelGGL((route_place_kernel<2, true>), dim3(chunks), dim3(kPlaceThreads), 0, st, a, (int)chunk);
    else hipLaunchKernelGGL((route_place_kernel<2, false>), dim3(chunks), dim3(kPlaceThreads), 0, st, a, (int)chunk);
    return hipGetLastError();
}

template <int LANES, int P>
static hipError_t launch_choose(const RouteArgs &a, hipStream_t st)
{
    return a.dtype == kF32 ? launch_of<LANES, P, kF32>(a, st) : a.dtype == kF16 ? launch_of<LANES, P, kF16>(a, st) : launch_of<LANES, P, kBf16>(a, st);
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
