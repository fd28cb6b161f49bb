// Products of 8-bit rows and 4-bit weights on many rows (see ffn_s4.hip for the mathematics): tiles of BM rows x BN weight rows whose operands go from memory straight
// into a ring of LDS stages of 128 * WK numbers of k, and from there into v_mfma_i32_32x32x32_i8.
//
// The weights are the instruction's second operand, so that a lane's sixteen sums are sixteen rows' of one output: one scale a lane makes a group's sums float32s,
// which are added up in registers.  A 16-byte block of weights is two operands (its lower and upper halves); the rows' pieces are read in the order that fits.
// The matrix cores take 32 cycles for an instruction, a conversion and a multiply-add of its 16 sums 128 cycles for each group: in groups of 128 numbers (four
// instructions) as much, so waves share a SIMD by twos and one's sums are scaled under the other's products.
// WK waves of a tile share its k axis, each with 128 numbers of a stage, and join their sums in LDS at the end.
#pragma once
#include "ffn_s4.h"

#include <type_traits>

namespace icnn {

namespace {

typedef __attribute__((address_space(3))) void LdsVoid;

#define FFN_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | 0x0F70 | (((n) >> 4) << 14))
#define FFN_WAIT_LGKM() __builtin_amdgcn_s_waitcnt(0xC07F)

// Row q's 16-byte piece c lies at c ^ row_key(q) in its stage: sixteen lanes read the same piece of rows 16 i + 0..15 and find them in sixteen different places of the
// 256 bytes that LDS hands out at a time
template <int BYTES>
__device__ __forceinline__ int row_key(int q)
{
    return BYTES == 64 ? (q >> 2) & 3 : BYTES == 128 ? (q >> 1) & 7 : q & 15;
}

template <int TN, int TM, int WN, int WM, int WK, int GROUP, bool GATED>
struct S4Tile {
    static constexpr int NW = WN * WM * WK, THREADS = NW * 64, BN = 32 * TN * WN, BM = 32 * TM * WM, XR = 128 * WK, WR = 64 * WK, STAGES = 3, STAGE = BM * XR + BN * WR;
    static constexpr int STEPS = WK == 1 ? 4 : 1, GROUPS = XR * STEPS / GROUP;     // of a chunk of scales, which come in together
    static constexpr int SCALES = GROUPS * BN * 4, LDS = STAGES * STAGE + 2 * SCALES + BM * 4, OUT = GATED ? BN / 2 : BN;
    static_assert(WM * 32 * OUT * 4 <= STAGES * STAGE && (WK - 1) * BM * BN * 4 <= STAGES * STAGE && LDS <= 163840, "what takes the ring's place");
};

}  // namespace

template <int TN, int TM, int WN, int WM, int WK, int GROUP, bool GATED, bool DIRECT, bool WIDE>
__global__ __launch_bounds__(WN * WM * WK * 64, 2) void s4_tiled_kernel(const LinearS4Args a, int tiles_n, int tiles_m, int per_xcd)
{
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-resource type exists in the device pass only
    typedef S4Tile<TN, TM, WN, WM, WK, GROUP, GATED> S;
    constexpr int NW = S::NW, BN = S::BN, BM = S::BM, XR = S::XR, WR = S::WR, STAGES = S::STAGES, STAGE = S::STAGE, STEPS = S::STEPS, GROUPS = S::GROUPS;
    constexpr int ROWS_W = 1024 / WR, ROWS_X = 1024 / XR, LW = BN / ROWS_W / NW, LX = BM / ROWS_X / NW, COPIES = LW + (DIRECT ? LX : 0);
    static_assert(LW * ROWS_W * NW == BN && LX * ROWS_X * NW == BM && (!GATED || TN % 2 == 0), "whole copies; a gate and its other layer in one wave");
    extern __shared__ __align__(1024) uint8_t lds[];
    float *const scales = (float *)(lds + STAGES * STAGE), *const row_scales = scales + 2 * GROUPS * BN;
    const int unit = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if (unit >= tiles_n * tiles_m) return;
    // eight rows of tiles, column after column: what an XCD has at one time shares its weights and rows
    constexpr int PANEL = 8;
    const int panel = unit / (PANEL * tiles_n), in_panel = unit - panel * PANEL * tiles_n, high = min(PANEL, tiles_m - panel * PANEL);
    const int tn0 = in_panel / high, tm0 = panel * PANEL + in_panel - tn0 * high;
    const int n0 = tn0 * S::OUT, m0 = tm0 * BM;

    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wk = wave % WK, wn = wave / WK % WN, wm = wave / (WK * WN);
    // weight row q of the tile: output of_row(q) from n0 on, of the second layer if second(q)
    auto of_row = [&](int q) { return GATED ? (q >> 6) * 32 + (q & 31) : q; };
    auto second = [&](int q) { return GATED && (q & 32); };

    // ---- copies: rows behind the last one are the last one again, pieces behind a row's end are out of the resource's range and arrive as zeros
    const __amdgpu_buffer_rsrc_t rs_w = __builtin_amdgcn_make_buffer_rsrc((void *)(a.w + n0 * a.ldw), 0, 0x7fffffff, 0x20000);
    const __amdgpu_buffer_rsrc_t rs_w2 = __builtin_amdgcn_make_buffer_rsrc((void *)((GATED ? a.w2 : a.w) + n0 * a.ldw), 0, 0x7fffffff, 0x20000);
    const int8_t *const x0 = a.x + m0 * a.ldx;
    const __amdgpu_buffer_rsrc_t rs_x = __builtin_amdgcn_make_buffer_rsrc((void *)x0, 0, 0x7fffffff, 0x20000);
    unsigned off_w[LW], off_x[LX];
    int piece_w[LW], piece_x[LX];
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int q = (j * NW + wave) * ROWS_W + lane / (WR / 16);
        piece_w[j] = 16 * ((lane % (WR / 16)) ^ row_key<WR>(q));
        off_w[j] = (unsigned)min(of_row(q), a.N - 1 - n0) * (unsigned)a.ldw + piece_w[j];
    }
#pragma unroll
    for (int j = 0; j < LX; ++j) {
        const int q = (j * NW + wave) * ROWS_X + lane / (XR / 16);
        piece_x[j] = 16 * ((lane % (XR / 16)) ^ row_key<XR>(q));
        off_x[j] = (unsigned)min(q, a.M - 1 - m0) * (unsigned)a.ldx + (DIRECT ? piece_x[j] : 0);
    }
    const int steps = (a.K + XR - 1) / XR;
    auto copy = [&](int s) {
        uint8_t *const to = lds + (s % STAGES) * STAGE + wave * 1024;
        const int left_w = (int)a.ldw - s * WR, left_x = a.K - s * XR;
#pragma unroll
        for (int j = 0; j < LW; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(second((j * NW + wave) * ROWS_W) ? rs_w2 : rs_w, (LdsVoid *)(to + BM * XR + j * NW * 1024), 16,
                                                     piece_w[j] < left_w ? off_w[j] : 0x80000000u, s * WR, 0, 0);
        if (DIRECT) {
#pragma unroll
            for (int j = 0; j < LX; ++j)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_x, (LdsVoid *)(to + j * NW * 1024), 16, piece_x[j] < left_x ? off_x[j] : 0x80000000u, s * XR, 0, 0);
        }
    };
    // rows that start anywhere, through registers
    v4i held[LX];
    auto fetch_rows = [&](int s) {
#pragma unroll
        for (int j = 0; j < LX; ++j) held[j] = *(const v4i_any *)(x0 + (off_x[j] + (unsigned)min(s * XR + piece_x[j], a.K - 16)));
    };
    auto put_rows = [&](int s) {
        uint8_t *const to = lds + (s % STAGES) * STAGE + wave * 1024 + lane * 16;
        const int left = a.K - s * XR;
        if (left < XR) {
#pragma unroll
            for (int j = 0; j < LX; ++j) held[j] = put_right(held[j], left - piece_x[j]);
        }
#pragma unroll
        for (int j = 0; j < LX; ++j) *(v4i *)(to + j * NW * 1024) = held[j];
    };

    // ---- scales: chunk c's are [group][weight row] in LDS, the next one's come in part by part under its steps.  Element e of a chunk is row e / GROUPS's of group
    // e % GROUPS: lanes next to each other read groups next to each other
    constexpr int PART = GROUPS * BN / STEPS, EACH = (PART + S::THREADS - 1) / S::THREADS;
    constexpr bool WHOLE = PART % S::THREADS == 0;
    uint32_t bits[EACH];
    auto fetch_scales = [&](int c, int part) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = part * PART + (WHOLE ? i * S::THREADS + t : min(i * S::THREADS + t, PART - 1)), q = e / GROUPS;
            const long long n = min(n0 + of_row(q), a.N - 1);
            bits[i] = scale_bits<WIDE>(second(q) ? a.ws2 : a.ws, n * a.groups + min(c * GROUPS + e % GROUPS, a.groups - 1));
        }
    };
    auto put_scales = [&](int c, int part) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = part * PART + i * S::THREADS + t;
            if (WHOLE || i * S::THREADS + t < PART)
                scales[((c & 1) * GROUPS + e % GROUPS) * BN + e / GROUPS] = c * GROUPS + e % GROUPS < a.groups ? scale_of(bits[i], a.scale_dtype) : 0.f;
        }
    };
    auto barrier = [&]() {
        FFN_WAIT_LGKM();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // ---- a stage's products
    const int r = lane & 31, h = lane >> 5;
    float sum[TN][TM][16] = {};
    auto products = [&](int s, int in_chunk, int c) {
        const uint8_t *const xs = lds + (s % STAGES) * STAGE, *const ws = xs + BM * XR;
        const float *const at = scales + (c & 1) * GROUPS * BN + wn * TN * 32 + r;
        auto rows = [&](int j, int piece) {
            const int q = (wm * TM + j) * 32 + r;
            return *(const v4i *)(xs + q * XR + (((wk * 8 + piece) ^ row_key<XR>(q)) << 4));
        };
        auto block = [&](int i, int b) {
            const int q = (wn * TN + i) * 32 + r;
            return *(const v4i *)(ws + q * WR + (((wk * 4 + b) ^ row_key<WR>(q)) << 4));
        };
        const int group0 = (in_chunk * WK + wk) * 128 / GROUP;
        auto scaled = [&](float(&to)[16], const v16i &acc, float scale) {
#pragma unroll
            for (int e = 0; e < 16; ++e) to[e] += (float)acc[e] * scale;
        };
        if constexpr (GROUP == 32) {                       // a block, its halves by the lanes' halves
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                v4i x[TM];
#pragma unroll
                for (int j = 0; j < TM; ++j) x[j] = rows(j, 2 * b + h);
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    const v4i from = block(i, b);
                    const float scale = at[(group0 + b) * BN + i * 32];
                    v4i w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = (int)((unsigned)from[e] << (h ? 0 : 4) & 0xf0f0f0f0u);
#pragma unroll
                    for (int j = 0; j < TM; ++j) scaled(sum[i][j], __builtin_amdgcn_mfma_i32_32x32x32_i8(x[j], w, v16i{}, 0, 0, 0), scale);
                }
            }
        } else {                                           // 64 numbers, a block in each half of the lanes: its lower and then its upper numbers
            constexpr int PAIRS = GROUP == 64 ? 1 : 2;     // of which a unit of the sums is made (a group of 256 is two units)
#pragma unroll
            for (int u = 0; u < 2 / PAIRS; ++u) {
                v4i x[TM][PAIRS][2];
#pragma unroll
                for (int j = 0; j < TM; ++j)
#pragma unroll
                    for (int p = 0; p < PAIRS; ++p)
#pragma unroll
                        for (int f = 0; f < 2; ++f) x[j][p][f] = rows(j, 4 * (u * PAIRS + p) + 2 * h + f);
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    v4i w[PAIRS][2];
#pragma unroll
                    for (int p = 0; p < PAIRS; ++p) {
                        const v4i from = block(i, 2 * (u * PAIRS + p) + h);
                        w[p][0] = sixteen_of<false>(from);
                        w[p][1] = sixteen_of<true>(from);
                    }
                    const float scale = at[(group0 + u) * BN + i * 32];
#pragma unroll
                    for (int j = 0; j < TM; ++j) {
                        v16i acc = {};
#pragma unroll
                        for (int p = 0; p < PAIRS; ++p)
#pragma unroll
                            for (int f = 0; f < 2; ++f) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[j][p][f], w[p][f], acc, 0, 0, 0);
                        scaled(sum[i][j], acc, scale);
                    }
                }
            }
        }
    };

    // ---- the stages in turn.  Behind a step's barrier all have done with the stage of the step before: the copies of two steps on go there.
    if (!DIRECT) {
        fetch_rows(0);
        put_rows(0);
        fetch_rows(1);
        put_rows(1);
    }
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
        fetch_scales(0, u);
        put_scales(0, u);
    }
    copy(0);
    copy(1);
    for (int i = t; i < BM; i += S::THREADS) row_scales[i] = a.xs[min(m0 + i, a.M - 1)];
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
        const int c = s / STEPS, part = s % STEPS;
        FFN_WAIT_VMCNT(COPIES);                            // (the next step's are still in flight; others that are make this wait for more)
        barrier();
        fetch_scales(c + 1, part);
        if (!DIRECT) fetch_rows(s + 2);
        copy(s + 2);
        products(s, part, c);
        if (!DIRECT) put_rows(s + 2);
        put_scales(c + 1, part);
    }
    FFN_WAIT_VMCNT(0);

    // ---- sums of one k range, by the waves of the first one
    barrier();
    if (WK > 1) {
        v4f *const part = (v4f *)lds;
        auto place = [&](int k, int i, int j, int e) { return ((((k - 1) * WN * WM + wm * WN + wn) * TN + i) * TM + j) * 256 + e * 64 + lane; };
        if (wk > 0) {
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[place(wk, i, j, e)] = v4f{sum[i][j][4 * e], sum[i][j][4 * e + 1], sum[i][j][4 * e + 2], sum[i][j][4 * e + 3]};
        }
        barrier();
        if (wk == 0) {
#pragma unroll
            for (int k = 1; k < WK; ++k)
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int j = 0; j < TM; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const v4f p = part[place(k, i, j, e)];
#pragma unroll
                            for (int q = 0; q < 4; ++q) sum[i][j][4 * e + q] += p[q];
                        }
        }
        barrier();
    }

    // ---- epilogue, 32 rows of each wave at a time: a lane finishes sixteen rows of an output, up to the residual, and leaves them in LDS; then a thread has eight
    // outputs of a row, whose residual and y are read and written in whole lines
    constexpr int OUT = S::OUT, TPR = OUT / 8, PASS = S::THREADS / TPR, ROUND = WM * 32, PASSES = (ROUND + PASS - 1) / PASS;
    float *const out = (float *)lds;
    auto column = [&](int q, int c) { return q * OUT + (OUT >= 64 ? c ^ ((q >> 2 & 1) << 5) : c); };
    const int o = 8 * (t % TPR), n = n0 + o;
    auto finish = [&](auto dt) {
        constexpr int DT = dt, ITEM = DT == kF32 ? 4 : 2;
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            Eight<DT> res[PASSES] = {};
            auto row = [&](int p) { return t / TPR + p * PASS; };          // of the round's; row_at: of the tile's
            auto row_at = [&](int q) { return (q / 32 * TM + j) * 32 + q % 32; };
            auto there = [&](int p) { return row(p) < ROUND && m0 + row_at(row(p)) < a.M && n < a.N; };
            if (!GATED && a.res) {
#pragma unroll
                for (int p = 0; p < PASSES; ++p)
                    if (there(p)) {
                        const uint8_t *const from = (const uint8_t *)a.res + ((m0 + row_at(row(p))) * a.ldr + n) * ITEM;
                        res[p] = n + 8 <= a.N ? load_eight<DT>(from, 0) : load_up_to_eight<DT>(from, a.N - n);
                    }
            }
            if (wk == 0) {
                float xs[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) xs[e] = row_scales[(wm * TM + j) * 32 + 8 * (e >> 2) + 4 * h + (e & 3)];
#pragma unroll
                for (int i = 0; i < TN; i += GATED ? 2 : 1) {
                    const int col = of_row((wn * TN + i) * 32 + r), at = min(n0 + col, a.N - 1);
                    const float b1 = a.bias ? a.bias[at] : 0.f, b2 = GATED && a.bias2 ? a.bias2[at] : 0.f;
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = sum[i][j][e] * xs[e] + b1;
                    activate_all(v, a.act, DT);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        if (GATED) v[e] *= sum[i + (GATED ? 1 : 0)][j][e] * xs[e] + b2;
                        out[column(wm * 32 + 8 * (e >> 2) + 4 * h + (e & 3), col)] = v[e];
                    }
                }
            }
            barrier();
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int q = row(p);
                if (!there(p)) continue;
                const v4f lo = *(const v4f *)(out + column(q, o)), hi = *(const v4f *)(out + column(q, o) + 4);
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                if (!GATED && a.res) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += value_of<DT>(res[p], e);
                }
                uint8_t *const to = (uint8_t *)a.y + ((m0 + row_at(q)) * a.ldy + n) * ITEM;
                if (n + 8 <= a.N) {
                    store_eight<DT>(to, 0, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (n + e < a.N) store_number(to, e, DT, v[e]);
                }
            }
            if (j + 1 < TM) barrier();
        }
    };
    if (a.dtype == kBf16) finish(std::integral_constant<int, kBf16>{});
    else if (a.dtype == kF16) finish(std::integral_constant<int, kF16>{});
    else finish(std::integral_constant<int, kF32>{});
#endif
}

template <int TN, int TM, int WN, int WM, int WK, int GROUP, bool GATED, bool DIRECT, bool WIDE>
static hipError_t launch_s4_one(const LinearS4Args &a, hipStream_t st)
{
    typedef S4Tile<TN, TM, WN, WM, WK, GROUP, GATED> S;
    const int tiles_n = (a.N + S::OUT - 1) / S::OUT, tiles_m = (a.M + S::BM - 1) / S::BM;
    const long long per = ((long long)tiles_n * tiles_m + 7) / 8;
    if (!fits_launch(per * 8, S::THREADS)) return hipErrorInvalidValue;
    auto *const k = s4_tiled_kernel<TN, TM, WN, WM, WK, GROUP, GATED, DIRECT, WIDE>;
    if (hipError_t e = allow_large_lds((const void *)k)) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)(per * 8)), dim3(S::THREADS), S::LDS, st, a, tiles_n, tiles_m, (int)per);
    return hipGetLastError();
}

template <int TN, int TM, int WN, int WM, int WK, int GROUP, bool GATED>
static hipError_t launch_s4_tile(const LinearS4Args &a, hipStream_t st)
{
    const bool wide = a.scale_dtype == kF32, direct = ((uintptr_t)a.x & 15) == 0 && ((a.ldx | a.K) & 15) == 0;
    if (direct) return wide ? launch_s4_one<TN, TM, WN, WM, WK, GROUP, GATED, true, true>(a, st) : launch_s4_one<TN, TM, WN, WM, WK, GROUP, GATED, true, false>(a, st);
    return wide ? launch_s4_one<TN, TM, WN, WM, WK, GROUP, GATED, false, true>(a, st) : launch_s4_one<TN, TM, WN, WM, WK, GROUP, GATED, false, false>(a, st);
}

// (the tiles in the order of kS4Tiles)
template <int GROUP>
static hipError_t launch_s4_tiles(const LinearS4Args &a, int tile, hipStream_t st)
{
    if (a.w2) {
        switch (tile) {
        case 0: return launch_s4_tile<2, 2, 4, 2, 1, GROUP, true>(a, st);
        case 1: return launch_s4_tile<2, 2, 2, 2, 2, GROUP, true>(a, st);
        default: return launch_s4_tile<2, 1, 1, 2, 4, GROUP, true>(a, st);
        }
    }
    switch (tile) {
    case 0: return launch_s4_tile<2, 2, 4, 2, 1, GROUP, false>(a, st);
    case 1: return launch_s4_tile<2, 2, 2, 2, 2, GROUP, false>(a, st);
    default: return launch_s4_tile<1, 1, 1, 2, 4, GROUP, false>(a, st);
    }
}

}  // namespace icnn
