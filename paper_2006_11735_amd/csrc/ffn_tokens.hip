// Products of up to four 8-bit rows and weights (see ffn_linear.hip for the mathematics): the single tokens of a decoder.  Nothing but the weights' way from memory
// counts.  A wave reads whole kilobytes of a weight row an instruction (16 bytes a lane), all of its rows' in flight at once, against the rows' pieces that it
// keeps in registers; sums are taken four products an instruction (v_dot4) and joined over the lanes at the end, over the KW waves that share the k axis in LDS.
// 1 x 16384 -> 4096: 12.4 us (5.4 TB/s), 1 x 4096 -> 16384: 11.9, gated 1 x 4096 -> 16384: 21.3 (6.3 TB/s); 4 rows: 14.1, 13.1 and 22.2.
#include "ffn_common.h"

namespace icnn {

namespace {

// The sums over a wave's lanes of V numbers (a power of two) of every lane: number lane / (64 / V) is returned.  While there are two numbers left each half of
// the lanes takes one of them, so that a step's additions halve: V - 1 of them and the rest of the six, where V sums by themselves take 6 V.
template <int V>
__device__ __forceinline__ int sums_of_lanes(int (&s)[V])
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
            const int a = s[i], b = s[halve ? i + n : i];
            if (bit >= 4) {
                const auto r = bit == 5 ? __builtin_amdgcn_permlane32_swap(a, b, false, false) : __builtin_amdgcn_permlane16_swap(a, b, false, false);
                s[i] = (int)r[0] + (int)r[1];
            } else {
                const int mine = lane >> bit & 1 ? b : a, other = lane >> bit & 1 ? a : b;
                s[i] = mine + (bit == 3   ? __builtin_amdgcn_update_dpp(0, other, 0x140, 0xf, 0xf, true)      // sixteen lanes mirrored
                               : bit == 2 ? __builtin_amdgcn_update_dpp(0, other, 0x141, 0xf, 0xf, true)      // eight lanes mirrored
                               : bit == 1 ? __builtin_amdgcn_update_dpp(0, other, 0x4E, 0xf, 0xf, true)       // lanes ^ 2
                                          : __builtin_amdgcn_update_dpp(0, other, 0xB1, 0xf, 0xf, true));     // lanes ^ 1
            }
        }
    }
    return s[0];
}

}  // namespace

// MR rows; C kilobytes of k a wave, KW waves along k; OUT outputs a wave
template <int MR, int C, int KW, int OUT, bool GATED>
__global__ __launch_bounds__(64 * (KW > 4 ? KW : 4)) void linear_tokens_kernel(const LinearArgs a)
{
    constexpr int L = GATED ? 2 : 1, NW = KW > 4 ? KW : 4, V = OUT * L * MR;
    __shared__ int part[NW][V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = ((int)blockIdx.x * (NW / KW) + wave / KW) * OUT;      // (may lie behind the last output: nothing is stored then)
    // the pieces' places in a row, no further on than its last 16 bytes
    int at[C], left[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int k = ((wave % KW) * C + c) * 1024 + 16 * lane;
        left[c] = a.K - k;
        at[c] = min(k, a.K - 16);
    }
    v4i x[MR][C], w[OUT][L][C];
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x[m][c] = *(const v4i_any *)(a.x + min(m, a.M - 1) * a.ldx + at[c]);
        }
#pragma unroll
    for (int b = 0; b < OUT; ++b)
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
            for (int c = 0; c < C; ++c)
                w[b][l][c] = __builtin_nontemporal_load((const v4i_any *)((l ? a.w2 : a.w) + min(n0 + b, a.N - 1) * a.ldw + at[c]));
    // what the lane that will finish output j % OUT of row j / OUT needs
    const int fm = min(lane / OUT, a.M - 1), fn = min(n0 + lane % OUT, a.N - 1);
    const bool finishes = lane < OUT * MR && wave % KW == 0 && lane / OUT < a.M && n0 + lane % OUT < a.N;
    float xs = 0.f, s1 = 0.f, b1 = 0.f, s2 = 0.f, b2 = 0.f;
    uint32_t res = 0;
    if (finishes) {
        xs = a.xs[fm];
        s1 = a.ws[fn];
        if (a.bias) b1 = a.bias[fn];
        if (GATED) {
            s2 = a.ws2[fn];
            if (a.bias2) b2 = a.bias2[fn];
        } else if (a.res) {
            res = load_bits(a.res, fm * a.ldr + fn, a.dtype);
        }
    }
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int c = 0; c < C; ++c) x[m][c] = last_of(x[m][c], left[c]);
    int sum[V] = {};
#pragma unroll
    for (int b = 0; b < OUT; ++b)
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
            for (int m = 0; m < MR; ++m)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[(m * OUT + b) * L + l] = __builtin_amdgcn_sdot4(w[b][l][c][e], x[m][c][e], sum[(m * OUT + b) * L + l], false);
    const int s = sums_of_lanes(sum);
    if (lane % (64 / V) == 0) part[wave][lane / (64 / V)] = s;
    __syncthreads();
    if (finishes) {
        int c1 = 0, c2 = 0;
#pragma unroll
        for (int q = 0; q < KW; ++q) {
            c1 += part[wave + q][lane * L];
            if (GATED) c2 += part[wave + q][lane * L + 1];
        }
        float v[1] = {(float)c1 * xs * s1 + b1};
        activate_all(v, a.act, a.dtype);
        if (GATED) v[0] *= (float)c2 * xs * s2 + b2;
        else if (a.res) v[0] += value_of(res, a.dtype);
        store_number(a.y, fm * a.ldy + fn, a.dtype, v[0]);
    }
}

template <int MR, int C, int KW, int OUT>
static void launch_tokens(const LinearArgs &a, hipStream_t st)
{
    constexpr int NW = KW > 4 ? KW : 4;
    const dim3 grid((unsigned)((a.N + OUT * (NW / KW) - 1) / (OUT * (NW / KW)))), block(64 * NW);
    if (a.w2) {
        constexpr int HALF = OUT / 2 < 1 ? 1 : OUT / 2;
        const dim3 wide((unsigned)((a.N + HALF * (NW / KW) - 1) / (HALF * (NW / KW))));
        hipLaunchKernelGGL((linear_tokens_kernel<MR, C, KW, HALF, true>), wide, block, 0, st, a);
    } else {
        hipLaunchKernelGGL((linear_tokens_kernel<MR, C, KW, OUT, false>), grid, block, 0, st, a);
    }
}

// A kilobyte of k a wave, the waves of a workgroup along k: by fewer waves with more of a row each 1 x 4096 -> 16384 takes 12.3 us instead of 11.7, 4 x 4096 ->
// 16384 14.6 instead of 12.9, 4 x 32768 -> 2048 18 instead of 14.4
template <int MR>
static void launch_rows_of(const LinearArgs &a, hipStream_t st)
{
    if (a.K <= 1024) launch_tokens<MR, 1, 1, 4>(a, st);
    else if (a.K <= 2048) launch_tokens<MR, 1, 2, 8>(a, st);
    else if (a.K <= 4096) launch_tokens<MR, 1, 4, 8>(a, st);
    else if (a.K <= 8192) launch_tokens<MR, 1, 8, 4>(a, st);
    else if (a.K <= 16384) launch_tokens<MR, 1, 16, 4>(a, st);
    else launch_tokens<MR, 2, 16, 4>(a, st);
}

hipError_t launch_tokens_linear(const LinearArgs &a, hipStream_t st)
{
    if (a.M == 1) launch_rows_of<1>(a, st);
    else if (a.M == 2) launch_rows_of<2>(a, st);
    else launch_rows_of<4>(a, st);
    return hipGetLastError();
}

}  // namespace icnn
