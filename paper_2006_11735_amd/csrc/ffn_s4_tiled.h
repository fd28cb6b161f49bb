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
    static constexpr int NW = WN * WM * WK, THREADS = NW * 64, BN = 32 * TN * WN, BM = 32 * TM * WM, XR = 128 * WK, WR = 64 * WK, STAGE = BM * XR + BN * WR;
    static constexpr int STEPS = WK == 1 ? (GROUP == 32 ? 2 : 4) : 1, GROUPS = XR * STEPS / GROUP;       // of a chunk of scales, which come in together
    static constexpr int SCALES = GROUPS * BN * 4, REST = 2 * SCALES + BM * 4, STAGES = 4 * STAGE + REST <= 163840 ? 4 : 3, LDS = STAGES * STAGE + REST;
    static constexpr bool AHEAD = STAGES == 4;             // fragments of the next stage under this one's products
    static constexpr int OUT = GATED ? BN / 2 : BN;
    static_assert(WM * 32 * OUT * 4 <= STAGES * STAGE && (WK - 1) * BM * BN * 4 <= STAGES * STAGE && LDS <= 163840 && THREADS == kS4TileThreads, "what takes the ring's place");
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
    // (no branch on whether a row ends in the step: behind one the compiler no longer counts the copies in flight and waits for them where it waits for the scales)
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

    // ---- scales: chunk c's are [group][weight row] in LDS, the next one's on their way.  Element e of a chunk is row e / GROUPS's of group e % GROUPS: lanes next to each
    // other read groups next to each other
    constexpr int EACH = (GROUPS * BN + S::THREADS - 1) / S::THREADS;
    constexpr bool WHOLE = GROUPS * BN % S::THREADS == 0;
    uint32_t bits[EACH];
    auto fetch_scales = [&](int c) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = WHOLE ? i * S::THREADS + t : min(i * S::THREADS + t, GROUPS * BN - 1), q = e / GROUPS;
            const long long n = min(n0 + of_row(q), a.N - 1);
            bits[i] = scale_bits<WIDE>(second(q) ? a.ws2 : a.ws, n * a.groups + min(c * GROUPS + e % GROUPS, a.groups - 1));
        }
    };
    auto put_scales = [&](int c) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = i * S::THREADS + t;
            if (WHOLE || e < GROUPS * BN)
                scales[((c & 1) * GROUPS + e % GROUPS) * BN + e / GROUPS] = c * GROUPS + e % GROUPS < a.groups ? scale_of(bits[i], a.scale_dtype) : 0.f;
        }
    };
    auto barrier = [&]() {
        FFN_WAIT_LGKM();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // ---- a stage's products.  A unit is what one scale holds for, 128 numbers at most (a group of 256 is two): a tile of 32 x 32 sums takes `CHAIN` instructions for it,
    // and then 32 for the scaling, which is done under the next tile's products; the last tile's is under the next stage's.
    const int r = lane & 31, h = lane >> 5;
    constexpr int NUMBERS = GROUP < 128 ? GROUP : 128, UNITS = 128 / NUMBERS, CHAIN = NUMBERS / 32, TILES = UNITS * TN * TM, RAW = GROUP == 32 ? 1 : CHAIN / 2;
    typedef float v16f __attribute__((ext_vector_type(16)));
    v16f sum[TN][TM] = {};
    v16i last = {};                                        // the last tile's sums of the stage before, and their scale
    float behind = 0.f;
    v4i x[TM][CHAIN], raw[TN][RAW];
    float scale[TN];
    // Fragments of unit u of stage s: of a unit of 32 numbers lane half h has the weights' block's half h, of others the block h of each two, of which first the lower
    // and then the upper numbers
    const int row_x = (wm * TM * 32 + r) * XR, row_w = BM * XR + (wn * TN * 32 + r) * WR;         // (32 rows on, the keys are the same)
    auto load_rows = [&](int j, int s, int u) {
        const uint8_t *const from = lds + (s % STAGES) * STAGE + j * 32 * XR;
#pragma unroll
        for (int f = 0; f < CHAIN; ++f) {
            const int piece = wk * 8 + (GROUP == 32 ? 2 * u + h : u * (NUMBERS / 16) + (f >> 1) * 4 + 2 * h + (f & 1));
            x[j][f] = *(const v4i *)(from + (row_x + ((piece ^ row_key<XR>(r)) << 4)));
        }
    };
    auto load_weights = [&](int i, int s, int u) {
        const uint8_t *const from = lds + (s % STAGES) * STAGE + i * 32 * WR;
#pragma unroll
        for (int p = 0; p < RAW; ++p) {
            const int piece = wk * 4 + (GROUP == 32 ? u : u * (NUMBERS / 32) + 2 * p + h);
            raw[i][p] = *(const v4i *)(from + (row_w + ((piece ^ row_key<WR>(r)) << 4)));
        }
    };
    auto load_scale = [&](int i, int s, int u) {
        scale[i] = scales[((s / STEPS & 1) * GROUPS + (s % STEPS * WK + wk) * 128 / GROUP + u) * BN + (wn * TN + i) * 32 + r];
    };
    auto load_first = [&](int s) {
#pragma unroll
        for (int j = 0; j < (TM > 1 ? TM - 1 : 1); ++j) load_rows(j, s, 0);
#pragma unroll
        for (int i = 0; i < TN; ++i) load_weights(i, s, 0);
    };
    // What a unit's first tile needs is read under the unit before, also that of the stage before if that one's copies can be waited for so early; its last rows under its
    // own first tile
    auto products = [&](int s) {
        asm volatile("s_nop 15\n\ts_nop 3" : "+v"(last));       // (see mfma_drain in conv_common.h: their products are behind the loop's branch)
        v16i before = last;
        v4i w[CHAIN];
        if (!S::AHEAD) load_first(s);
#pragma unroll
        for (int q = 0; q < TILES; ++q) {
            const int u = q / (TN * TM), i = q / TM % TN, j = q % TM;
            const int next = u + 1 < UNITS ? s : s + 1, unit = u + 1 < UNITS ? u + 1 : 0;
            const int v = (q + TILES - 1) % TILES;         // the tile before
            v16f &to = sum[v / TM % TN][v % TM];
            const float by = q ? scale[v / TM % TN] : behind;
            if (i == 0 && j == 0 && TM > 1) load_rows(TM - 1, s, u);
            if (j == 0) {
#pragma unroll
                for (int p = 0; p < RAW; ++p) {
                    if (GROUP == 32) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[0][e] = (int)((unsigned)raw[i][p][e] << (h ? 0 : 4) & 0xf0f0f0f0u);
                    } else {
                        w[2 * p] = sixteen_of<false>(raw[i][p]);
                        w[(2 * p + 1) % CHAIN] = sixteen_of<true>(raw[i][p]);
                    }
                }
                load_scale(i, s, u);
                if (S::AHEAD || u + 1 < UNITS) load_weights(i, next, unit);
            }
            // The empty statements keep the order: an instruction of this tile's, a part of the tile before's sums to scale under it.  Without them the compiler puts
            // all products first, whose sums are more than there are registers.
            v16i t = {};
            asm volatile("" : "+v"(before));
#pragma unroll
            for (int f = 0; f < CHAIN; ++f) {
                t = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[j][f], w[f], t, 0, 0, 0);
                asm volatile("" : "+v"(t));
#pragma unroll
                for (int e = 0; e < 16 / CHAIN; ++e) to[16 / CHAIN * f + e] += (float)before[16 / CHAIN * f + e] * by;
                asm volatile("" : "+v"(to));
            }
            before = t;
            if (i == TN - 1 && (j < TM - 1 || TM == 1) && (S::AHEAD || u + 1 < UNITS)) load_rows(j, next, unit);
            __builtin_amdgcn_sched_barrier(0x194);         // (what computes stays in its tile; memory's instructions may move)
        }
        last = before;
        behind = scale[TN - 1];
    };

    // ---- the stages in turn.  Behind a step's barrier all have done with the stage of the step before: the copies of STAGES - 1 steps on go there.  The step's have
    // arrived by then (AHEAD: the next one's).
    if (!DIRECT) {
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) {
            fetch_rows(s);
            put_rows(s);
        }
    }
    fetch_scales(0);
    put_scales(0);
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) copy(s);
    for (int i = t; i < BM; i += S::THREADS) row_scales[i] = a.xs[min(m0 + i, a.M - 1)];
    if (S::AHEAD) {
        asm volatile("" ::: "memory");
        FFN_WAIT_VMCNT((STAGES - 2) * COPIES);
        barrier();
        load_first(0);
    }
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
        const int c = s / STEPS, part = s % STEPS;
        asm volatile("" ::: "memory");
        FFN_WAIT_VMCNT((S::AHEAD ? STAGES - 3 : STAGES - 2) * COPIES);     // (later ones are still in flight; others that are make this wait for more)
        barrier();
        if (part == 0) fetch_scales(c + 1);
        if (!DIRECT) fetch_rows(s + STAGES - 1);
        copy(s + STAGES - 1);
        products(s);
        if (!DIRECT) put_rows(s + STAGES - 1);
        if (part == STEPS - 1) put_scales(c + 1);
    }
    FFN_WAIT_VMCNT(0);
    asm volatile("s_nop 15\n\ts_nop 3" : "+v"(last));
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[TN - 1][TM - 1][e] += (float)last[e] * behind;

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
    case 2: return launch_s4_tile<1, 1, 1, 2, 4, GROUP, false>(a, st);
    default: return launch_s4_tile<1, 1, 1, 1, 8, GROUP, false>(a, st);
    }
}

}  // namespace icnn
