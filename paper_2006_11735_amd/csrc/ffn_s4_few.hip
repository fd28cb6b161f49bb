// Products of few 8-bit rows and 4-bit weights (see ffn_s4.hip for the mathematics).  What counts is how fast the weights come in: each is used for 16 * MT rows
// at most.  A workgroup has 16 T outputs of all rows (16 of a gated layer, see launch_group); its eight waves share the k axis, in turns of RB bytes of a weight row (twice as many numbers), and join their sums in
// LDS at the end.  A wave's weights come in whole lines, a turn ahead in registers, and go through LDS, where no other wave reads them, into the order of the matrix
// instruction: 64 numbers of k, of which lane l has 16 (half (l >> 4) & 1 of block l >> 5).  The rows, which every workgroup reads, come out of the caches, a turn ahead too.
#include "ffn_s4.h"

#include <type_traits>

namespace icnn {

namespace {

// Eight waves of T * 16 rows of weights (both layers' sixteen, where there are two); with 32 of them the rows come from the caches half as often as with 16
constexpr int NW = 8, RB = 128, PIECES = RB / 16, COPIES = RB / 64, XQ = RB / 32;

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

// What a wave's lanes write to LDS others of it read: the hardware keeps a wave's order, the compiler knows of one lane's own addresses only
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }

}  // namespace

template <int MT, int T, int GROUP, bool GATED, bool WIDE>
__global__ __launch_bounds__(NW * 64, 2) void s4_few_kernel(const LinearS4Args a)
{
    constexpr int L = GATED ? 2 : 1, NT = T / L;           // layers, 16 outputs each of the workgroup
    constexpr int GROUPS = 2 * RB / GROUP, SCALES = (16 * GROUPS + 63) / 64;       // groups a turn; scales a lane brings
    constexpr int WEIGHTS = NW * T * 16 * RB, SCALE_BYTES = NW * T * GROUPS * 64, PART = NW * MT * T * 1024;
    __shared__ __align__(16) uint8_t lds[WEIGHTS + SCALE_BYTES > PART ? WEIGHTS + SCALE_BYTES : PART];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * (16 * NT), row_bytes = (int)a.ldw;
    const int turns = (row_bytes + RB - 1) / RB, mine = wave < turns ? (turns - wave + NW - 1) / NW : 0;        // this wave's turns: wave, wave + NW, ...

    uint8_t *const weights = lds + wave * (T * 16 * RB);
    float *const scales = (float *)(lds + WEIGHTS) + wave * (T * GROUPS * 16);

    // Tile u of the weights: outputs n0 + 16 u .. of the one layer, or layer u's n0 ...  Copy i of a turn has the rows i * 1024 / RB + lane * 16 / RB; a row's 16-byte
    // piece c lies at c ^ (row % PIECES)
    const uint8_t *from[T][COPIES];
    int piece[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int q = (i * 1024 + lane * 16) / RB;
        piece[i] = 16 * ((lane % PIECES) ^ (q % PIECES));
#pragma unroll
        for (int u = 0; u < T; ++u) from[u][i] = (GATED && u ? a.w2 : a.w) + min(n0 + (GATED ? 0 : 16 * u) + q, a.N - 1) * a.ldw;
    }
    v4i held[T][COPIES];
    uint32_t held_scales[T][SCALES];
    // (a piece behind the row's end is its last one: the rows' numbers there are zeros)
    auto fetch = [&](int t) {
        const int at = min(wave + t * NW, turns - 1) * RB;
#pragma unroll
        for (int u = 0; u < T; ++u) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) held[u][i] = __builtin_nontemporal_load((const v4i *)(from[u][i] + min(at + piece[i], row_bytes - 16)));
#pragma unroll
            for (int i = 0; i < SCALES; ++i) {             // number j is row j / GROUPS's of group j % GROUPS
                const int j = min(64 * i + lane, 16 * GROUPS - 1), n = min(n0 + (GATED ? 0 : 16 * u) + j / GROUPS, a.N - 1);
                held_scales[u][i] = scale_bits<WIDE>(GATED && u ? a.ws2 : a.ws, (long long)n * a.groups + min(2 * at / GROUP + j % GROUPS, a.groups - 1));
            }
        }
    };
    auto put = [&](int t) {
        const int first = 2 * (wave + t * NW) * RB / GROUP;
#pragma unroll
        for (int u = 0; u < T; ++u) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) *(v4i *)(weights + u * (16 * RB) + i * 1024 + lane * 16) = held[u][i];
#pragma unroll
            for (int i = 0; i < SCALES; ++i) {
                const int j = 64 * i + lane;
                if (16 * GROUPS % 64 == 0 || j < 16 * GROUPS)
                    scales[(u * GROUPS + j % GROUPS) * 16 + j / GROUPS] = first + j % GROUPS < a.groups ? scale_of(held_scales[u][i], a.scale_dtype) : 0.f;
            }
        }
    };
    const int8_t *x[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = a.x + min(16 * i + r, a.M - 1) * a.ldx;
    v4i xv[MT][XQ];
    auto load_rows = [&](int t, int q) {                   // their piece q of turn t
        const int k0 = min(wave + t * NW, turns - 1) * RB * 2;
#pragma unroll
        for (int i = 0; i < MT; ++i) xv[i][q] = load_there(x[i], k0 + 64 * q + 16 * g, a.K);
    };
    float sum[MT][T][4] = {};
    // (a piece of the rows is loaded for the next turn as soon as it has been used: one set of registers)
    auto turn = [&](int t, auto more) {
        put(t);
        in_order();
        if (more) fetch(t + 1);
        const int k0 = (wave + t * NW) * RB * 2;
        if (k0 + 2 * RB > a.K) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < XQ; ++q) xv[i][q] = put_right(xv[i][q], a.K - k0 - 64 * q - 16 * g);
        }
        v4i acc[T][MT] = {};
        auto scaled = [&](v4i(&c)[MT], int u, int i) {     // group i's sums are whole
            const v4f s = *(const v4f *)&scales[(u * GROUPS + i) * 16 + 4 * g];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[m][u][e] += (float)c[m][e] * s[e];
#pragma unroll
            for (int m = 0; m < MT; ++m) c[m] = v4i{};
        };
#pragma unroll
        for (int q = 0; q < XQ; ++q) {
#pragma unroll
            for (int u = 0; u < T; ++u) {
                const int c = 2 * q + (g >> 1);
                const v4i block = *(const v4i *)(weights + u * (16 * RB) + r * RB + ((c ^ (r % PIECES)) << 4));
                v4i w, w2, other[MT] = {};
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (int)((unsigned)block[e] << (g & 1 ? 0 : 4) & 0xf0f0f0f0u);
                if (GROUP == 32) {                         // the two blocks' sums by themselves
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w2[e] = g > 1 ? w[e] : 0;
                        w[e] = g > 1 ? 0 : w[e];
                    }
#pragma unroll
                    for (int m = 0; m < MT; ++m) other[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w2, xv[m][q], other[m], 0, 0, 0);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[u][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, xv[m][q], acc[u][m], 0, 0, 0);
                if (GROUP == 32) {
                    drain(acc[u]);
                    drain(other);
                    scaled(acc[u], u, 2 * q);
                    scaled(other, u, 2 * q + 1);
                } else if ((q + 1) % (GROUP / 64) == 0) {
                    drain(acc[u]);
                    scaled(acc[u], u, q / (GROUP / 64));
                }
            }
            if (more) load_rows(t + 1, q);
        }
        in_order();
    };
    if (mine) {
        fetch(0);
#pragma unroll
        for (int q = 0; q < XQ; ++q) load_rows(0, q);
        for (int t = 0; t + 1 < mine; ++t) turn(t, std::true_type{});
        turn(mine - 1, std::false_type{});
    }
    __syncthreads();                                       // (the sums go where weights and scales have been)
    v4f *const part = (v4f *)lds;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int u = 0; u < T; ++u) part[((wave * MT + i) * T + u) * 64 + lane] = v4f{sum[i][u][0], sum[i][u][1], sum[i][u][2], sum[i][u][3]};
    __syncthreads();
    // wave i finishes the rows 16 (i / NT) + 0..15 of outputs 16 (i % NT) + 0..15: a lane has four outputs of a row
    if (wave < MT * NT) {
        const int i = wave / NT, u = wave % NT;
        float s[4] = {}, s2[4] = {};
#pragma unroll
        for (int q = 0; q < NW; ++q) {
            const v4f c = part[((q * MT + i) * T + u) * 64 + lane], c2 = part[((q * MT + i) * T + u + L - 1) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] += c[e];
                if (GATED) s2[e] += c2[e];
            }
        }
        const int m = 16 * i + r;
        if (m < a.M) finish_four_s4<GATED>(a, s, s2, m, n0 + 16 * u + 4 * g);
    }
}

template <int MT, int T, int GROUP, bool GATED>
static void launch_of(const LinearS4Args &a, hipStream_t st)
{
    constexpr int PER = GATED ? 8 * T : 16 * T;
    const dim3 grid((unsigned)((a.N + PER - 1) / PER)), block(NW * 64);
    if (a.scale_dtype == kF32) hipLaunchKernelGGL((s4_few_kernel<MT, T, GROUP, GATED, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((s4_few_kernel<MT, T, GROUP, GATED, false>), grid, block, 0, st, a);
}

// Sixteen outputs a workgroup where those are no more than there are compute units (24 rows, 4096 -> 4096 7.6 us, with 32 outputs 8.3; 2048 -> 5461 8.8 and 6.5, 8192 -> 8192
// 20.2 and 14.7)
template <int MT, int GROUP>
static void launch_group(const LinearS4Args &a, hipStream_t st)
{
    if (a.w2) launch_of<MT, 2, GROUP, true>(a, st);
    else if (a.N <= 16 * 256) launch_of<MT, 1, GROUP, false>(a, st);
    else launch_of<MT, 2, GROUP, false>(a, st);
}

template <int MT>
static void launch_rows(const LinearS4Args &a, hipStream_t st)
{
    switch (a.group) {
    case 32: return launch_group<MT, 32>(a, st);
    case 64: return launch_group<MT, 64>(a, st);
    case 128: return launch_group<MT, 128>(a, st);
    default: return launch_group<MT, 256>(a, st);
    }
}

hipError_t launch_few_s4(const LinearS4Args &a, hipStream_t st)
{
    if (a.M <= 16) launch_rows<1>(a, st);
    else launch_rows<2>(a, st);
    return hipGetLastError();
}

}  // namespace icnn
