// Products of up to four 8-bit rows and 4-bit weights (see ffn_s4.hip for the mathematics): the single tokens of a decoder.  Nothing but the weights' way from memory
// counts.  A wave reads a kilobyte of a weight row an instruction, 2048 numbers, a block of 32 a lane and all of its rows' in flight at once, against the rows' pieces
// that it keeps in registers; the block's sum, by v_dot4, is exact, its scale makes it a float32, and those are joined over the lanes and over the KW waves that share
// the k axis.
#include "ffn_s4.h"

namespace icnn {

namespace {

// The sums over a wave's lanes of V numbers (a power of two) of every lane: number lane / (64 / V) is returned.  While there are two numbers left each half of
// the lanes takes one of them (sums_of_lanes in ffn_tokens.h, of floats)
__device__ __forceinline__ float moved(float v, int control)
{
    const int b = __builtin_bit_cast(int, v);
    const int r = control == 3   ? __builtin_amdgcn_update_dpp(0, b, 0x140, 0xf, 0xf, true)      // sixteen lanes mirrored
                  : control == 2 ? __builtin_amdgcn_update_dpp(0, b, 0x141, 0xf, 0xf, true)      // eight lanes mirrored
                  : control == 1 ? __builtin_amdgcn_update_dpp(0, b, 0x4E, 0xf, 0xf, true)       // lanes ^ 2
                                 : __builtin_amdgcn_update_dpp(0, b, 0xB1, 0xf, 0xf, true);      // lanes ^ 1
    return __builtin_bit_cast(float, r);
}

template <int V>
__device__ __forceinline__ float sums_of_lanes(float (&s)[V])
{
    const int lane = threadIdx.x & 63;
    int n = V;
#pragma unroll
    for (int bit = 5; bit >= 0; --bit) {
        const bool halve = n > 1;
        if (halve) n /= 2;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (i >= n) continue;
            const float a = s[i], b = s[halve ? i + n : i];
            if (bit >= 4) {
                const unsigned ua = __builtin_bit_cast(unsigned, a), ub = __builtin_bit_cast(unsigned, b);
                const auto r = bit == 5 ? __builtin_amdgcn_permlane32_swap(ua, ub, false, false) : __builtin_amdgcn_permlane16_swap(ua, ub, false, false);
                const unsigned r0 = r[0], r1 = r[1];
                s[i] = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
            } else {
                const float mine = lane >> bit & 1 ? b : a, other = lane >> bit & 1 ? a : b;
                s[i] = mine + moved(other, bit);
            }
        }
    }
    return s[0];
}

}  // namespace

// MR rows; KW waves along k; OUT outputs a wave; WIDE: scales of four bytes
template <int MR, int KW, int OUT, bool GATED, bool WIDE>
__global__ __launch_bounds__(64 * (KW > 4 ? KW : 4)) void s4_tokens_kernel(const LinearS4Args a)
{
    constexpr int L = GATED ? 2 : 1, NW = KW > 4 ? KW : 4, V = OUT * L * MR;
    __shared__ float part[NW][V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = ((int)blockIdx.x * (NW / KW) + wave / KW) * OUT;      // (may lie behind the last output: nothing is stored then)
    const int block = (wave % KW) * 64 + lane, at = min(block, (int)(a.ldw / kBlockBytes) - 1), k = block * kBlockNumbers, group = min(k / a.group, a.groups - 1);
    v4i x[MR][2], w[OUT][L];
    uint32_t bits[OUT][L];
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) x[m][h] = load_there(a.x + min(m, a.M - 1) * a.ldx, k + 16 * h, a.K);
#pragma unroll
    for (int b = 0; b < OUT; ++b)
#pragma unroll
        for (int l = 0; l < L; ++l) {
            const int n = min(n0 + b, a.N - 1);
            w[b][l] = __builtin_nontemporal_load((const v4i *)((l ? a.w2 : a.w) + n * a.ldw) + at);
            bits[b][l] = scale_bits<WIDE>(l ? a.ws2 : a.ws, (long long)n * a.groups + group);
        }
    // what the lane that will finish output lane % OUT of row lane / OUT needs
    const int fm = min(lane / OUT, a.M - 1), fn = min(n0 + lane % OUT, a.N - 1);
    const bool finishes = lane < OUT * MR && wave % KW == 0 && lane / OUT < a.M && n0 + lane % OUT < a.N;
    float xs = 0.f, b1 = 0.f, b2 = 0.f;
    uint32_t res = 0;
    if (finishes) {
        xs = a.xs[fm];
        if (a.bias) b1 = a.bias[fn];
        if (GATED) {
            if (a.bias2) b2 = a.bias2[fn];
        } else if (a.res) {
            res = load_bits(a.res, fm * a.ldr + fn, a.dtype);
        }
    }
    if (((wave % KW) + 1) * 64 * kBlockNumbers > a.K) {    // (the wave that has the row's end, and those behind it)
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) x[m][h] = put_right(x[m][h], a.K - k - 16 * h);
    }
    float sum[V];
#pragma unroll
    for (int b = 0; b < OUT; ++b)
#pragma unroll
        for (int l = 0; l < L; ++l) {
            const v4i low = sixteen_of<false>(w[b][l]), high = sixteen_of<true>(w[b][l]);
            const float scale = k < a.K ? scale_of(bits[b][l], a.scale_dtype) : 0.f;
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                int dot = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dot = __builtin_amdgcn_sdot4(low[e], x[m][0][e], dot, false);
                    dot = __builtin_amdgcn_sdot4(high[e], x[m][1][e], dot, false);
                }
                sum[(m * OUT + b) * L + l] = (float)dot * scale;
            }
        }
    const float s = sums_of_lanes(sum);
    if (lane % (64 / V) == 0) part[wave][lane / (64 / V)] = s;
    __syncthreads();
    if (finishes) {
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int q = 0; q < KW; ++q) {
            c1 += part[wave + q][lane * L];
            if (GATED) c2 += part[wave + q][lane * L + 1];
        }
        float v[1] = {c1 * xs + b1};
        activate_all(v, a.act, a.dtype);
        if (GATED) v[0] *= c2 * xs + b2;
        else if (a.res) v[0] += value_of(res, a.dtype);
        store_number(a.y, fm * a.ldy + fn, a.dtype, v[0]);
    }
}

template <int MR, int KW, int OUT, bool GATED>
static void launch_of(const LinearS4Args &a, hipStream_t st)
{
    constexpr int NW = KW > 4 ? KW : 4, PER = OUT * (NW / KW);
    const dim3 grid((unsigned)((a.N + PER - 1) / PER)), block(64 * NW);
    if (a.scale_dtype == kF32) hipLaunchKernelGGL((s4_tokens_kernel<MR, KW, OUT, GATED, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((s4_tokens_kernel<MR, KW, OUT, GATED, false>), grid, block, 0, st, a);
}

template <int MR, int KW, int OUT>
static void launch_waves(const LinearS4Args &a, hipStream_t st)
{
    if (a.w2) launch_of<MR, KW, OUT / 2, true>(a, st);
    else launch_of<MR, KW, OUT, false>(a, st);
}

template <int MR>
static void launch_rows(const LinearS4Args &a, hipStream_t st)
{
    if (a.K <= 2048) launch_waves<MR, 1, 8>(a, st);
    else if (a.K <= 4096) launch_waves<MR, 2, 8>(a, st);
    else if (a.K <= 8192) launch_waves<MR, 4, 8>(a, st);
    else if (a.K <= 16384) launch_waves<MR, 8, 8>(a, st);
    else launch_waves<MR, 16, 4>(a, st);
}

hipError_t launch_tokens_s4(const LinearS4Args &a, hipStream_t st)
{
    if (a.M == 1) launch_rows<1>(a, st);
    else if (a.M == 2) launch_rows<2>(a, st);
    else launch_rows<4>(a, st);
    return hipGetLastError();
}

}  // namespace icnn
