// Products of 8-bit rows and weights on few rows (see ffn_linear.hip for the mathematics).  What counts is how fast the weights come in: each is used for
// 16 * MT rows at most.  A workgroup has 16 outputs of all rows; its NW waves share the k axis, in turns of 256 bytes, and join their sums in LDS at the end.  A wave's
// weights go from memory into a ring of LDS stages of its own (no other wave reads them, so its own wait is all the synchronisation), 256 bytes of a weight
// row by sixteen lanes; the rows, which every workgroup reads, come out of the caches into registers, a turn ahead.  Bound by the weights' way and by the rows', which
// grows with their number: 8192 -> 8192 on 8 rows 4.6 TB/s, on 16 3.7; 32 rows, gated 4096 -> 8192 3.6 TB/s.
#include "ffn_common.h"

#include <type_traits>

namespace icnn {

namespace {

typedef __attribute__((address_space(3))) void LdsVoid;

#define FFN_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | 0x0F70 | (((n) >> 4) << 14))

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

// Four waves of two stages: with eight, or more stages, fewer workgroups share a compute unit and less of one's start and end is under the others' copies
// (16 rows, 4096 -> 4096: 6.3 us, with eight waves 7.4 to 8.2; turns of 512 bytes 8.2)
constexpr int NW = kFewWaves, DEPTH = 2, RB = kFewTurn;

}  // namespace

template <int MT, bool GATED, bool DIRECT>
__global__ __launch_bounds__(NW * 64) void linear_few_kernel(const LinearArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-resource type exists in the device pass only
    constexpr int L = GATED ? 2 : 1, WB = 16 * RB, STAGE = L * WB, CP = WB / 1024, COPIES = CP * L, XQ = RB / 64, XL = XQ * MT;
    extern __shared__ __align__(1024) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16;
    uint8_t *const ring = lds + wave * (DEPTH * STAGE);
    const int turns = (a.K + RB - 1) / RB, mine = wave < turns ? (turns - wave + NW - 1) / NW : 0;      // this wave's turns: wave, wave + NW, ...

    // ---- weights: copy i of a stage has the rows 4 i + lane / 16; a row's 16-byte piece c lies at c ^ row, so that sixteen lanes that read the same piece of
    // sixteen rows find them in sixteen different places of 256 bytes
    const __amdgpu_buffer_rsrc_t rs[2] = {__builtin_amdgcn_make_buffer_rsrc((void *)(a.w + n0 * a.ldw), 0, 0x7fffffff, 0x20000),
                                          __builtin_amdgcn_make_buffer_rsrc((void *)((GATED ? a.w2 : a.w) + n0 * a.ldw), 0, 0x7fffffff, 0x20000)};
    unsigned off[CP];
    int piece[CP];
#pragma unroll
    for (int i = 0; i < CP; ++i) {
        const int q = (i * 1024 + lane * 16) / RB;
        piece[i] = (lane % (RB / 16)) ^ q;
        off[i] = (unsigned)min(q, a.N - 1 - n0) * (unsigned)a.ldw + 16 * piece[i];
    }
    auto copy = [&](int t) {                               // the wave's turn t; behind the last one nothing but zeros comes
        const int k0 = (wave + t * NW) * RB, left = t < mine ? a.K - k0 : 0;
        uint8_t *const to = ring + (t % DEPTH) * STAGE;
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
            for (int i = 0; i < CP; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs[l], (LdsVoid *)(to + l * WB + i * 1024), 16, 16 * piece[i] < left ? off[i] : 0x80000000u, k0, 0, 2);      // (2: not to be kept)
    };
    // the same through registers, for rows that start anywhere (no load hangs on a condition, behind which the compiler would wait for all loads in flight)
    v4i held[COPIES];
    auto fetch = [&](int t) {
        const int k0 = (wave + t * NW) * RB;
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
            for (int i = 0; i < CP; ++i)
                held[CP * l + i] = *(const v4i_any *)((l ? a.w2 : a.w) + n0 * a.ldw + (off[i] + (unsigned)min(k0, a.K - 16 - 16 * piece[i])));
    };
    auto put = [&](int t) {
#pragma unroll
        for (int c = 0; c < COPIES; ++c) *(v4i *)(ring + (t % DEPTH) * STAGE + c * 1024 + lane * 16) = held[c];
    };

    const int8_t *x[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = a.x + min(16 * i + r, a.M - 1) * a.ldx;
    v4i xv[2][MT][XQ];
    auto load_rows = [&](int t, int set) {                 // (behind the last turn the row's last 16 numbers, which nothing multiplies)
        const int k0 = min(wave + t * NW, turns) * RB;
        if (k0 + RB <= a.K) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < XQ; ++q) xv[set][i][q] = *(const v4i_any *)(x[i] + k0 + 64 * q + 16 * g);
        } else {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < XQ; ++q) {
                    const int k = k0 + 64 * q + 16 * g;
                    xv[set][i][q] = *(const v4i_any *)(x[i] + min(k, a.K - 16));
                }
        }
    };

    if (DIRECT) {
#pragma unroll
        for (int t = 0; t < DEPTH - 1; ++t) copy(t);
    } else if (mine) {
        fetch(0);
    }
    Four<GATED> f;                                         // of the rows 16 wave + 0..15, which this wave finishes
    if (wave < MT) load_four<GATED>(a, min(16 * wave + r, a.M - 1), n0 + 4 * g, f);
    v4i acc[MT * L] = {};
    auto turn = [&](int t, auto set) {
        load_rows(t + 1, 1 - set);
        if (DIRECT) {
            copy(t + DEPTH - 1);                           // into the stage that the last turn has read (its fragments have left it)
            asm volatile("" ::: "memory");
            FFN_WAIT_VMCNT(XL + COPIES);                   // all but the next turn's rows and weights (tests/test_few_waits.py counts them in the built kernels)
            asm volatile("" ::: "memory");
        } else {
            put(t);
            fetch(t + 1);
            const int k0 = (wave + t * NW) * RB;
            if (k0 + RB > a.K) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int q = 0; q < XQ; ++q) xv[set][i][q] = last_of(xv[set][i][q], a.K - k0 - 64 * q - 16 * g);
            }
        }
        const uint8_t *const from = ring + (t % DEPTH) * STAGE + r * RB;
#pragma unroll
        for (int q = 0; q < XQ; ++q)
#pragma unroll
            for (int l = 0; l < L; ++l) {
                const v4i wv = *(const v4i *)(from + l * WB + (((4 * q + g) ^ r) << 4));
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i * L + l] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv[set][i][q], acc[i * L + l], 0, 0, 0);
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    if (mine) load_rows(0, 0);
    for (int t = 0; t < mine; t += 2) {
        turn(t, std::integral_constant<int, 0>{});
        if (t + 1 < mine) turn(t + 1, std::integral_constant<int, 1>{});
    }
    if (DIRECT) FFN_WAIT_VMCNT(0);
    drain(acc);
    __syncthreads();
    v4i *const part = (v4i *)lds;
#pragma unroll
    for (int i = 0; i < MT * L; ++i) part[(wave * MT * L + i) * 64 + lane] = acc[i];
    __syncthreads();
    // wave i finishes the rows 16 i + 0..15: a lane has four outputs of one
    if (wave < MT) {
        v4i c = part[wave * L * 64 + lane], c2 = part[(wave * L + L - 1) * 64 + lane];
#pragma unroll
        for (int q = 1; q < NW; ++q) {
            c += part[((q * MT + wave) * L) * 64 + lane];
            if (GATED) c2 += part[((q * MT + wave) * L + 1) * 64 + lane];
        }
        const int m = 16 * wave + r;
        if (m < a.M) finish_four<GATED>(a, c, c2, f, m, n0 + 4 * g);
    }
#endif
}

template <int MT, bool GATED, bool DIRECT>
static hipError_t launch_one(const LinearArgs &a, hipStream_t st)
{
    constexpr int L = GATED ? 2 : 1, RING = NW * DEPTH * L * 16 * RB, PART = NW * MT * L * 1024, LDS = RING > PART ? RING : PART;
    static_assert(LDS <= 65536, "no more than a kernel may have unasked");
    hipLaunchKernelGGL((linear_few_kernel<MT, GATED, DIRECT>), dim3((unsigned)((a.N + 15) / 16)), dim3(NW * 64), LDS, st, a);
    return hipGetLastError();
}

template <int MT>
static hipError_t launch_few(const LinearArgs &a, hipStream_t st)
{
    const bool direct = (((uintptr_t)a.w | (uintptr_t)a.w2) & 15) == 0 && ((a.ldw | a.K) & 15) == 0;
    if (direct) return a.w2 ? launch_one<MT, true, true>(a, st) : launch_one<MT, false, true>(a, st);
    return a.w2 ? launch_one<MT, true, false>(a, st) : launch_one<MT, false, false>(a, st);
}

hipError_t launch_few_linear(const LinearArgs &a, hipStream_t st)
{
    return a.M <= 16 ? launch_few<1>(a, st) : a.M <= 32 ? launch_few<2>(a, st) : launch_few<4>(a, st);
}

}  // namespace icnn
