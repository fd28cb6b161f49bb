// Products of 8-bit rows and weights on many rows (see ffn_linear.hip for the mathematics): tiles of BM rows x BN weight rows whose operands go from memory
// straight into a ring of LDS stages of BK bytes of k, and from there into v_mfma_i32_32x32x32_i8.
//
// The weights are the instruction's first operand, so that a lane's sixteen sums belong to one row m and, by the order in which the weight rows are
// handed to it, to sixteen outputs n next to each other: the epilogue reads scales, biases and residual and writes y in whole 16-byte pieces.
// In a gated layer the 32-row groups of a tile's weights are gate and up in turn, so a wave holds both sums of an output in the same lane and register.
#include "ffn_common.h"

namespace icnn {

namespace {

typedef __attribute__((address_space(3))) void LdsVoid;

#define FFN_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | 0x0F70 | (((n) >> 4) << 14))
#define FFN_WAIT_LGKM() __builtin_amdgcn_s_waitcnt(0xC07F)

struct TiledArgs {
    LinearArgs l;
    int tiles_n, tiles_m, per_xcd;
};

// Where row q's 16-byte piece c lies in its stage.  Eight lanes that read the same piece of eight rows, as the fragments of either operand have them (rows
// 8 i + 0..7, or of the weights 0..3 and 16..19), find them in eight different pieces of the 128 bytes that LDS hands out together.
template <int BK, bool WEIGHTS>
__device__ __forceinline__ int piece_key(int q)
{
    if (BK == 128) return WEIGHTS ? (q & 3) | ((q >> 4) & 1) << 2 : q & 7;
    return WEIGHTS ? ((q >> 1) & 1) | ((q >> 4) & 1) << 1 : (q >> 1) & 3;
}

template <int TN, int TM>
__device__ __forceinline__ void drain(v16i (&acc)[TN][TM])
{
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) asm volatile("" : "+v"(acc[i][j]));
    asm volatile("s_nop 15\n\ts_nop 3");
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) asm volatile("" : "+v"(acc[i][j]));
}

}  // namespace

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED>
__global__ __launch_bounds__(WN * WM * 64, 1) void linear_tiled_kernel(const TiledArgs ta)
{
    constexpr int NW = WN * WM, BN = 32 * TN * WN, BM = 32 * TM * WM, ROWS = 1024 / BK, PIECES = BK / 16, SLICES = BK / 32;
    constexpr int LW = BN / ROWS / NW, LX = BM / ROWS / NW, LOADS = LW + LX, STAGE = (BN + BM) * BK, LDS_GROUPS = STAGES * STAGE / 4096;
    static_assert(LW * ROWS * NW == BN && LX * ROWS * NW == BM && SLICES >= 2 && SLICES % 2 == 0, "whole copies, two fragment sets in turn");
    extern __shared__ __align__(1024) uint8_t lds[];
    const LinearArgs &a = ta.l;
    const int slot = (int)(blockIdx.x & 7) * ta.per_xcd + (int)(blockIdx.x >> 3);
    if (slot >= ta.tiles_n * ta.tiles_m) return;
    // eight rows of tiles, column after column: what an XCD has at one time shares its weights and rows
    constexpr int GROUP = 8;
    const int panel = slot / (GROUP * ta.tiles_n), in_panel = slot - panel * GROUP * ta.tiles_n, high = min(GROUP, ta.tiles_m - panel * GROUP);
    const int tn0 = in_panel / high, tm0 = panel * GROUP + in_panel - tn0 * high;
    const int n0 = tn0 * (GATED ? BN / 2 : BN), m0 = tm0 * BM;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wm = wave / WN;

    // ---- copies: one instruction takes ROWS rows of BK bytes (16 a lane).  Rows behind the last one are the last one again, pieces of k behind the end are
    // out of the resource's range and arrive as zeros.
    const __amdgpu_buffer_rsrc_t rs_w = __builtin_amdgcn_make_buffer_rsrc((void *)(a.w + n0 * a.ldw), 0, 0x7fffffff, 0x20000);
    const __amdgpu_buffer_rsrc_t rs_w2 = __builtin_amdgcn_make_buffer_rsrc((void *)((GATED ? a.w2 : a.w) + n0 * a.ldw), 0, 0x7fffffff, 0x20000);
    const __amdgpu_buffer_rsrc_t rs_x = __builtin_amdgcn_make_buffer_rsrc((void *)(a.x + m0 * a.ldx), 0, 0x7fffffff, 0x20000);
    unsigned off_w[LW], off_x[LX];
    int piece_w[LW], piece_x[LX];
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int q = (j * NW + wave) * ROWS + lane / PIECES;
        piece_w[j] = (lane % PIECES) ^ piece_key<BK, true>(q);
        const int n = GATED ? (q >> 6) * 32 + (q & 31) : q;
        off_w[j] = (unsigned)min(n, a.N - 1 - n0) * (unsigned)a.ldw + 16 * piece_w[j];
    }
#pragma unroll
    for (int j = 0; j < LX; ++j) {
        const int q = (j * NW + wave) * ROWS + lane / PIECES;
        piece_x[j] = (lane % PIECES) ^ piece_key<BK, false>(q);
        off_x[j] = (unsigned)min(q, a.M - 1 - m0) * (unsigned)a.ldx + 16 * piece_x[j];
    }
    const int steps = (a.K + BK - 1) / BK;
    auto copy_step = [&](int s) {
        uint8_t *const to = lds + (s % STAGES) * STAGE + wave * 1024;
        const int k0 = s * BK;
        const bool whole = k0 + BK <= a.K;
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const unsigned off = whole || k0 + 16 * piece_w[j] < a.K ? off_w[j] : 0x80000000u;
            const bool up = GATED && (((j * NW + wave) * ROWS) & 32);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(up ? rs_w2 : rs_w, (LdsVoid *)(to + j * NW * 1024), 16, off, k0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < LX; ++j) {
            const unsigned off = whole || k0 + 16 * piece_x[j] < a.K ? off_x[j] : 0x80000000u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_x, (LdsVoid *)(to + BN * BK + j * NW * 1024), 16, off, k0, 0, 0);
        }
    };

    // ---- fragments: lane l has row l % 32 of its group and the 16 bytes l / 32 of a slice of 32.  Weight row r of a group is n = 16 ((r >> 2) & 1) +
    // 4 (r >> 3) + (r & 3), which makes register i of a lane in half h output 16 h + i.
    const int r = lane & 31, half = lane >> 5;
    const int qw = wn * TN * 32 + 16 * ((r >> 2) & 1) + 4 * (r >> 3) + (r & 3), qx = wm * TM * 32 + r;
    const int at_w = qw * BK + ((half ^ piece_key<BK, true>(qw)) << 4), at_x = BN * BK + qx * BK + ((half ^ piece_key<BK, false>(qx)) << 4);
    v4i fw[2][TN], fx[2][TM];
    auto read_slice = [&](int stage, int kk, int set) {
        const uint8_t *const from = lds + stage * STAGE;
#pragma unroll
        for (int i = 0; i < TN; ++i) fw[set][i] = *(const v4i *)(from + (at_w ^ (kk << 5)) + i * 32 * BK);
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[set][i] = *(const v4i *)(from + (at_x ^ (kk << 5)) + i * 32 * BK);
    };
    v16i acc[TN][TM] = {};
    auto multiply = [&](int set) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[set][i], fx[set][j], acc[i][j], 0, 0, 0);
    };

#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < steps) copy_step(s);
    if (steps >= STAGES) FFN_WAIT_VMCNT((STAGES - 1) * LOADS);
    else FFN_WAIT_VMCNT(0);
    __builtin_amdgcn_s_barrier();
    read_slice(0, 0, 0);
    // A stage's last slice is multiplied behind the barrier: its fragments have left LDS in front of it, so the stage is free for the copies issued there,
    // and the first fragments of the next one come in under those products.
    for (int s = 0; s < steps; ++s) {
#pragma unroll
        for (int kk = 0; kk < SLICES - 1; ++kk) {
            read_slice(s % STAGES, kk + 1, (kk + 1) & 1);
            multiply(kk & 1);
        }
        if (s + 1 < steps) {
            if (s + STAGES <= steps) FFN_WAIT_VMCNT((STAGES - 2) * LOADS);      // (the stages behind the next one are still in flight)
            else FFN_WAIT_VMCNT(0);
            FFN_WAIT_LGKM();
            __builtin_amdgcn_s_barrier();
            if (s + STAGES < steps) copy_step(s + STAGES);
            read_slice((s + 1) % STAGES, 0, 0);
        }
        multiply(1);
    }
    drain(acc);

    // ---- epilogue.  The sums go through LDS, every lane's own back to itself, only so that a loop can run over them: one body of code for all groups.
    constexpr int GROUPS = TN * TM, ROUND = LDS_GROUPS / NW < GROUPS ? LDS_GROUPS / NW : GROUPS;
    static_assert(GROUPS % ROUND == 0 && ROUND % TN == 0, "whole columns of groups a round");
    __syncthreads();
    uint8_t *const mine = lds + wave * ROUND * 4096 + lane * 16;
#pragma unroll
    for (int j0 = 0; j0 < TM; j0 += ROUND / TN) {
#pragma unroll
        for (int g = 0; g < ROUND; ++g)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v16i &c = acc[g % TN][j0 + g / TN];
                *(v4i *)(mine + g * 4096 + q * 1024) = v4i{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
            }
#pragma unroll 1
        for (int g = 0; g < ROUND; g += GATED ? 2 : 1) {
            const int i = g % TN, m = m0 + (wm * TM + j0 + g / TN) * 32 + r;
            const int n = n0 + (wn * TN + i) * (GATED ? 16 : 32) + 16 * half;
            int c[16], c2[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v4i t = *(const v4i *)(mine + g * 4096 + q * 1024), u = GATED ? *(const v4i *)(mine + (g + 1) * 4096 + q * 1024) : v4i{};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    c[4 * q + e] = t[e];
                    c2[4 * q + e] = u[e];
                }
            }
            if (m < a.M && n < a.N) finish_sixteen<GATED>(a, c, c2, m, n);
        }
    }
}

// Rows and weights that start at multiples of 16 bytes, with whole 16-byte pieces of k; a tile's rows within 2 GiB
bool tiled_linear_takes(const LinearArgs &a)
{
    const uintptr_t at = (uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.w2;
    return a.M > 64 && (at & 15) == 0 && ((a.ldx | a.ldw | a.K) & 15) == 0 && a.ldx <= (1 << 22) && a.ldw <= (1 << 22);
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED>
static hipError_t launch_tiles(const LinearArgs &a, hipStream_t st)
{
    constexpr int BN = 32 * TN * WN / (GATED ? 2 : 1), BM = 32 * TM * WM, LDS = 32 * (TN * WN + TM * WM) * BK * STAGES;
    TiledArgs t;
    t.l = a;
    t.tiles_n = (a.N + BN - 1) / BN;
    t.tiles_m = (a.M + BM - 1) / BM;
    const long long tiles = (long long)t.tiles_n * t.tiles_m, per = (tiles + 7) / 8;
    if (tiles > 0x7ffffff0LL) return hipErrorInvalidValue;
    t.per_xcd = (int)per;
    auto *const k = linear_tiled_kernel<TN, TM, WN, WM, BK, STAGES, GATED>;
    hipLaunchKernelGGL(k, dim3((unsigned)(per * 8)), dim3(WN * WM * 64), LDS, st, t);
    return hipGetLastError();
}

hipError_t launch_tiled_linear(const LinearArgs &a, hipStream_t st)
{
    return a.w2 ? launch_tiles<4, 4, 2, 2, 128, 2, true>(a, st) : launch_tiles<4, 4, 2, 2, 128, 2, false>(a, st);
}

}  // namespace icnn
