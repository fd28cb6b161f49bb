// Products of 8-bit rows and weights on few rows (see ffn_linear.hip for the mathematics).  What counts is how fast the weights come in: each is used for
// 16 * MT rows at most.  A workgroup has 16 outputs of all rows; its NW waves share the k axis, in turns of 128 bytes, take their weights from memory straight
// into the registers that v_mfma_i32_16x16x64_i8 reads (16 rows of 64 whole bytes an instruction), and join their sums in LDS.  The next turns' weights are
// on their way while the present ones are multiplied; the rows, which every workgroup reads, come out of the caches.
#include "ffn_common.h"

namespace icnn {

namespace {

// U turns of one operand's rows: 2 U pieces of 16 bytes a lane
template <int U>
__device__ __forceinline__ void load_turns(const int8_t *row, int first, int last, int step, v4i (&v)[2 * U])
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int8_t *const p = row + 128ll * min(first + u * step, last);      // (turns behind the last one are not multiplied)
        v[2 * u] = *(const v4i_any *)p;
        v[2 * u + 1] = *(const v4i_any *)(p + 64);
    }
}

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

template <int MT, int NW, int U, bool GATED>
__global__ __launch_bounds__(NW * 64) void linear_few_kernel(const LinearArgs a)
{
    constexpr int L = GATED ? 2 : 1;                       // products
    __shared__ v4i part[NW][MT * L][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
    const int8_t *w[L], *x[MT];
    w[0] = a.w + min(n0 + r, a.N - 1) * a.ldw + 16 * g;
    if (GATED) w[L - 1] = a.w2 + min(n0 + r, a.N - 1) * a.ldw + 16 * g;
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = a.x + min(m0 + 16 * i + r, a.M - 1) * a.ldx + 16 * g;

    Four<GATED> f;                                         // of the rows 16 wave + 0..15, which this wave finishes
    if (wave < MT) load_four<GATED>(a, min(m0 + 16 * wave + r, a.M - 1), n0 + 4 * g, f);
    v4i acc[MT * L] = {};
    auto multiply = [&](const v4i &wv, const v4i &xv, int i, int l) {
        acc[i * L + l] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, acc[i * L + l], 0, 0, 0);
    };
    const int turns = a.K >> 7;
    if (wave < turns) {
        v4i wv[2][L][2 * U];
#pragma unroll
        for (int l = 0; l < L; ++l) load_turns<U>(w[l], wave, turns - 1, NW, wv[0][l]);
        auto round = [&](int t, int set) {
            v4i xv[MT][2 * U];
#pragma unroll
            for (int i = 0; i < MT; ++i) load_turns<U>(x[i], t, turns - 1, NW, xv[i]);
            if (t + U * NW < turns) {
#pragma unroll
                for (int l = 0; l < L; ++l) load_turns<U>(w[l], t + U * NW, turns - 1, NW, wv[set ^ 1][l]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (t + u * NW < turns) {
#pragma unroll
                    for (int q = 2 * u; q < 2 * u + 2; ++q)
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int l = 0; l < L; ++l) multiply(wv[set][l][q], xv[i][q], i, l);
                }
        };
        for (int t = wave; t < turns; t += 2 * U * NW) {
            round(t, 0);
            if (t + U * NW < turns) round(t + U * NW, 1);
        }
    }
    if ((a.K & 127) && wave == turns % NW) {               // what is left of k
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int k = 128 * turns + 64 * q;
            if (k < a.K) {
                v4i wv[L];
#pragma unroll
                for (int l = 0; l < L; ++l) wv[l] = load_k16(w[l] - 16 * g, k + 16 * g, a.K);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const v4i xv = load_k16(x[i] - 16 * g, k + 16 * g, a.K);
#pragma unroll
                    for (int l = 0; l < L; ++l) multiply(wv[l], xv, i, l);
                }
            }
        }
    }
    drain(acc);
#pragma unroll
    for (int i = 0; i < MT * L; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    // wave i finishes the rows 16 i + 0..15: a lane has four outputs of one
    if (wave < MT) {
        const int m = m0 + 16 * wave + r, n = n0 + 4 * g;
        v4i c = part[0][wave * L][lane], c2 = part[0][wave * L + L - 1][lane];
#pragma unroll
        for (int q = 1; q < NW; ++q) {
            c += part[q][wave * L][lane];
            if (GATED) c2 += part[q][wave * L + 1][lane];
        }
        if (m < a.M) finish_four<GATED>(a, c, c2, f, m, n);
    }
}

bool few_linear_takes(const LinearArgs &a) { return a.M <= 64 * 65535LL; }

template <int MT, int NW, int U>
static void launch_few(const LinearArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * MT - 1) / (16 * MT))), block(NW * 64);
    if (a.w2) hipLaunchKernelGGL((linear_few_kernel<MT, NW, U, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((linear_few_kernel<MT, NW, U, false>), grid, block, 0, st, a);
}

hipError_t launch_few_linear(const LinearArgs &a, hipStream_t st)
{
    const int f = g_tuning.ff_few;
    if (f == 1) launch_few<1, 16, 2>(a, st);
    else if (f == 2) launch_few<1, 8, 2>(a, st);
    else if (f == 3) launch_few<1, 4, 4>(a, st);
    else if (f == 4) launch_few<1, 16, 4>(a, st);
    else if (f == 5) launch_few<2, 8, 1>(a, st);
    else if (f == 6) launch_few<2, 16, 1>(a, st);
    else if (f == 7) launch_few<4, 8, 1>(a, st);
    else if (f == 8) launch_few<4, 4, 2>(a, st);
    else if (a.M <= 16) launch_few<1, 8, 4>(a, st);
    else if (a.M <= 32) launch_few<2, 8, 2>(a, st);
    else launch_few<4, 8, 2>(a, st);
    return hipGetLastError();
}

}  // namespace icnn
