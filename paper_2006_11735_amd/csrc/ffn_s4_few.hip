// Products of few 8-bit rows and 4-bit weights (see ffn_s4.hip for the mathematics).  What counts is how fast the weights come in: each is used for 16 * MT rows
// at most.  A workgroup has 16 outputs of all rows; its four waves share the k axis, in turns of RB bytes of a weight row (twice as many numbers), and join their sums in
// LDS at the end.  A wave's weights come in whole lines, a turn ahead in registers, and go through LDS, where no other wave reads them, into the order of the matrix
// instruction: 64 numbers of k, of which lane l has 16 (half (l >> 4) & 1 of block l >> 5).  The rows, which every workgroup reads, come out of the caches, a turn ahead too.
#include "ffn_s4.h"

#include <type_traits>

namespace icnn {

namespace {

constexpr int NW = 4;

// Wait states between the last products and their sums' first reader (see mfma_drain in conv_common.h)
template <int N>
__device__ __forceinline__ void drain(v4i (&acc)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(acc[i]));
    asm volatile("s_nop 15\n\ts_nop 3");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(acc[i]));
}

}  // namespace

template <int MT, int GROUP, bool GATED, bool WIDE>
__global__ __launch_bounds__(NW * 64) void s4_few_kernel(const LinearS4Args a)
{
    constexpr int RB = MT == 4 ? 128 : 256, L = GATED ? 2 : 1, PIECES = RB / 16, COPIES = RB / 64, XQ = RB / 32;
    constexpr int GROUPS = 2 * RB / GROUP, SCALES = (16 * GROUPS + 63) / 64;       // groups a turn; scales a lane brings
    __shared__ __align__(16) uint8_t weights[NW][L][16 * RB];
    __shared__ __align__(16) float scales[NW][L][GROUPS * 16];
    __shared__ __align__(16) float part[NW][MT * L][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, row_bytes = (int)a.ldw;
    const int turns = (row_bytes + RB - 1) / RB, mine = wave < turns ? (turns - wave + NW - 1) / NW : 0;        // this wave's turns: wave, wave + NW, ...

    // copy i of a turn has the rows i * 1024 / RB + lane * 16 / RB; a row's 16-byte piece c lies at c ^ (row % PIECES)
    const uint8_t *from[COPIES];
    int piece[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int q = (i * 1024 + lane * 16) / RB;
        piece[i] = (lane % PIECES) ^ (q % PIECES);
        from[i] = a.w + min(n0 + q, a.N - 1) * a.ldw;
    }
    const long long second = GATED ? a.w2 - a.w : 0;
    v4i held[L * COPIES];
    uint32_t held_scales[L * SCALES];
    // (a piece behind the row's end is its last one: the rows' numbers there are zeros)
    auto fetch = [&](int t) {
        const int at = min(wave + t * NW, turns - 1) * RB;
#pragma unroll
        for (int l = 0; l < L; ++l) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i)
                held[l * COPIES + i] = __builtin_nontemporal_load((const v4i *)(from[i] + l * second + min(at + 16 * piece[i], row_bytes - 16)));
#pragma unroll
            for (int i = 0; i < SCALES; ++i) {             // number j is row j / GROUPS's of group j % GROUPS
                const int j = min(64 * i + lane, 16 * GROUPS - 1);
                held_scales[l * SCALES + i] = scale_bits<WIDE>(l ? a.ws2 : a.ws, (long long)min(n0 + j / GROUPS, a.N - 1) * a.groups + min(2 * at / GROUP + j % GROUPS, a.groups - 1));
            }
        }
    };
    auto put = [&](int t) {
        const int first = 2 * (wave + t * NW) * RB / GROUP;
#pragma unroll
        for (int l = 0; l < L; ++l) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) *(v4i *)(weights[wave][l] + i * 1024 + lane * 16) = held[l * COPIES + i];
#pragma unroll
            for (int i = 0; i < SCALES; ++i) {
                const int j = 64 * i + lane;
                if (16 * GROUPS % 64 == 0 || j < 16 * GROUPS)
                    scales[wave][l][j % GROUPS * 16 + j / GROUPS] = first + j % GROUPS < a.groups ? scale_of(held_scales[l * SCALES + i], a.scale_dtype) : 0.f;
            }
        }
    };
    const int8_t *x[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = a.x + min(16 * i + r, a.M - 1) * a.ldx;
    v4i xv[2][MT][XQ];
    auto load_rows = [&](int t, int set) {
        const int k0 = min(wave + t * NW, turns - 1) * RB * 2;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < XQ; ++q) xv[set][i][q] = load_there(x[i], k0 + 64 * q + 16 * g, a.K);
    };
    float sum[MT * L][4] = {};
    auto turn = [&](int t, auto set) {
        load_rows(t + 1, 1 - set);
        put(t);
        fetch(t + 1);
        const int k0 = (wave + t * NW) * RB * 2;
        if (k0 + 2 * RB > a.K) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < XQ; ++q) xv[set][i][q] = put_right(xv[set][i][q], a.K - k0 - 64 * q - 16 * g);
        }
#pragma unroll
        for (int l = 0; l < L; ++l) {
            v4i acc[MT] = {}, other[MT] = {};
            auto scaled = [&](v4i(&c)[MT], int i) {        // group i's sums are whole
                const v4f s = *(const v4f *)&scales[wave][l][i * 16 + 4 * g];
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[m * L + l][e] += (float)c[m][e] * s[e];
#pragma unroll
                for (int m = 0; m < MT; ++m) c[m] = v4i{};
            };
#pragma unroll
            for (int q = 0; q < XQ; ++q) {
                const int c = 2 * q + (g >> 1);
                const v4i block = *(const v4i *)(weights[wave][l] + r * RB + ((c ^ (r % PIECES)) << 4));
                v4i w, w2;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (int)((unsigned)block[e] << (g & 1 ? 0 : 4) & 0xf0f0f0f0u);
                if (GROUP == 32) {                         // the two blocks' sums by themselves
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w2[e] = g > 1 ? w[e] : 0;
                        w[e] = g > 1 ? 0 : w[e];
                    }
#pragma unroll
                    for (int m = 0; m < MT; ++m) other[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w2, xv[set][m][q], other[m], 0, 0, 0);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, xv[set][m][q], acc[m], 0, 0, 0);
                if (GROUP == 32) {
                    drain(acc);
                    drain(other);
                    scaled(acc, 2 * q);
                    scaled(other, 2 * q + 1);
                } else if ((q + 1) % (GROUP / 64) == 0) {
                    drain(acc);
                    scaled(acc, q / (GROUP / 64));
                }
            }
        }
    };
    if (mine) {
        fetch(0);
        load_rows(0, 0);
    }
    for (int t = 0; t < mine; t += 2) {
        turn(t, std::integral_constant<int, 0>{});
        if (t + 1 < mine) turn(t + 1, std::integral_constant<int, 1>{});
    }
#pragma unroll
    for (int i = 0; i < MT * L; ++i) *(v4f *)&part[wave][i][lane * 4] = v4f{sum[i][0], sum[i][1], sum[i][2], sum[i][3]};
    __syncthreads();
    // wave i finishes the rows 16 i + 0..15: a lane has four outputs of one
    if (wave < MT) {
        float s[4] = {}, s2[4] = {};
#pragma unroll
        for (int q = 0; q < NW; ++q) {
            const v4f c = *(const v4f *)&part[q][wave * L][lane * 4], c2 = *(const v4f *)&part[q][wave * L + L - 1][lane * 4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] += c[e];
                if (GATED) s2[e] += c2[e];
            }
        }
        const int m = 16 * wave + r;
        if (m < a.M) finish_four_s4<GATED>(a, s, s2, m, n0 + 4 * g);
    }
}

template <int MT, int GROUP>
static void launch_of(const LinearS4Args &a, hipStream_t st)
{
    const dim3 grid((unsigned)((a.N + 15) / 16)), block(NW * 64);
    const bool wide = a.scale_dtype == kF32;
    if (a.w2 && wide) hipLaunchKernelGGL((s4_few_kernel<MT, GROUP, true, true>), grid, block, 0, st, a);
    else if (a.w2) hipLaunchKernelGGL((s4_few_kernel<MT, GROUP, true, false>), grid, block, 0, st, a);
    else if (wide) hipLaunchKernelGGL((s4_few_kernel<MT, GROUP, false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((s4_few_kernel<MT, GROUP, false, false>), grid, block, 0, st, a);
}

template <int MT>
static void launch_rows(const LinearS4Args &a, hipStream_t st)
{
    switch (a.group) {
    case 32: return launch_of<MT, 32>(a, st);
    case 64: return launch_of<MT, 64>(a, st);
    case 128: return launch_of<MT, 128>(a, st);
    default: return launch_of<MT, 256>(a, st);
    }
}

hipError_t launch_few_s4(const LinearS4Args &a, hipStream_t st)
{
    if (a.M <= 16) launch_rows<1>(a, st);
    else if (a.M <= 32) launch_rows<2>(a, st);
    else launch_rows<4>(a, st);
    return hipGetLastError();
}

}  // namespace icnn
