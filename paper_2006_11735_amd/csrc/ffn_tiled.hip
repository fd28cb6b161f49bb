// Products of 8-bit rows and weights on many rows (see ffn_linear.hip for the mathematics): tiles of BM rows x BN weight rows whose operands go from memory
// straight into a ring of LDS stages of BK bytes of k, and from there into v_mfma_i32_32x32x32_i8.
//
// The weights are the instruction's first operand, so that a lane's sixteen sums belong to one row m and, by the order in which the weight rows are
// handed to it, to sixteen outputs n next to each other: the epilogue reads scales, biases and residual and writes y in whole 16-byte pieces.
// In a gated layer the 32-row groups of a tile's weights are gate and up in turn, so a wave holds both sums of an output in the same lane and register.
#include "ffn_common.h"

#include <type_traits>

namespace icnn {

namespace {

typedef __attribute__((address_space(3))) void LdsVoid;

#define FFN_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | 0x0F70 | (((n) >> 4) << 14))
#define FFN_WAIT_LGKM() __builtin_amdgcn_s_waitcnt(0xC07F)

struct TiledArgs {
    LinearArgs l;
    int tiles_n, tiles_m, per_xcd;
    // Split k: a tile's steps in `splits` ranges of `steps_per` (the last one may have fewer), each a workgroup of its own.  A range leaves its sums in `part`; the
    // one that arrives last at the tile's counter adds the others' and finishes the tile.  The sums are integers: the order of arrival changes nothing.
    int splits, steps_per;
    int32_t *part;
    unsigned *counters;            // zero before the launch and after it
};

// Row q's 16-byte piece c lies at c ^ piece_key(q) in its stage.  LDS hands out 256 bytes at a time, the pieces of sixteen lanes: those read the same piece of sixteen
// rows, as the fragments of either operand have them (rows 16 i + 0..15, of the weights 0..3, 16..19, 4..7, 20..23), and find them in sixteen different places
// of the 256 bytes.
template <int BK, bool WEIGHTS>
__device__ __forceinline__ int piece_key(int q)
{
    if (BK == 128) return WEIGHTS ? ((q >> 1) & 3) | ((q >> 4) & 1) << 2 : (q >> 1) & 7;
    return WEIGHTS ? ((q >> 2) & 1) | ((q >> 4) & 1) << 1 : (q >> 2) & 3;
}

// fn(0) ... fn(N - 1), the numbers as constants
template <int N, class F>
__device__ __forceinline__ void times(std::integral_constant<int, N>, F &&fn)
{
    if constexpr (N > 0) {
        times(std::integral_constant<int, N - 1>{}, fn);
        fn(std::integral_constant<int, N - 1>{});
    }
}

// Waves a SIMD when as many workgroups of `waves` waves as their LDS lets share a compute unit do (three at most: the registers are wanted too)
constexpr int waves_per_simd(int waves, int lds_bytes)
{
    const int groups = 163840 / lds_bytes < 3 ? 163840 / lds_bytes : 3;
    return groups * waves < 4 ? 1 : groups * waves / 4;
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

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
__global__ __launch_bounds__(WN * WM * 64, waves_per_simd(WN * WM, 32 * (TN * WN + TM * WM) * BK * STAGES)) void linear_tiled_kernel(const TiledArgs ta)
{
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-resource type exists in the device pass only
    constexpr int NW = WN * WM, BN = 32 * TN * WN, BM = 32 * TM * WM, ROWS = 1024 / BK, PIECES = BK / 16, SLICES = BK / 32;
    constexpr int LW = BN / ROWS / NW, LX = BM / ROWS / NW, LOADS = LW + LX, STAGE = (BN + BM) * BK;
    static_assert(DIRECT || STAGES == 2, "copies through registers are one stage ahead");
    static_assert(LW * ROWS * NW == BN && LX * ROWS * NW == BM && SLICES >= 2 && SLICES % 2 == 0, "whole copies, two fragment sets in turn");
    extern __shared__ __align__(1024) uint8_t lds[];
    const LinearArgs &a = ta.l;
    const int unit = (int)(blockIdx.x & 7) * ta.per_xcd + (int)(blockIdx.x >> 3);
    if (unit >= ta.tiles_n * ta.tiles_m * ta.splits) return;
    const int slot = unit / ta.splits, range = unit - slot * ta.splits;
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
    const int first = range * ta.steps_per * BK, steps = min(ta.steps_per, (a.K - first + BK - 1) / BK), end = min(a.K, first + steps * BK);
    // copies FROM .. TO - 1 of step s: of the weights, then of the rows.  Behind the last step nothing but zeros comes.
    auto copy_part = [&](int s, auto from, auto to) {
        uint8_t *const at = lds + (s % STAGES) * STAGE + wave * 1024;
        const int k0 = first + s * BK, left = end - k0;
#pragma unroll
        for (int j = from; j < to; ++j) {
            if (j < LW) {
                const bool up = GATED && (((j * NW + wave) * ROWS) & 32);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(up ? rs_w2 : rs_w, (LdsVoid *)(at + j * NW * 1024), 16, 16 * piece_w[j] < left ? off_w[j] : 0x80000000u, k0, 0, 0);
            } else {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_x, (LdsVoid *)(at + BN * BK + (j - LW) * NW * 1024), 16, 16 * piece_x[j - LW] < left ? off_x[j - LW] : 0x80000000u,
                                                         k0, 0, 0);
            }
        }
    };
    // The same through registers, for rows that start anywhere: the loads of AHEAD steps (as many as there are registers for) are in flight while a stage is multiplied,
    // put_step's stores follow.  No load hangs on a condition: the compiler then counts the loads in flight, behind a branch it would wait for all of them.  A piece
    // that goes beyond the row's end is its last 16 numbers, in both operands; put_step clears those of the rows' that have been before, or all behind the end.
    constexpr int AHEAD = DIRECT || TN * TM > 4 ? 1 : LOADS <= 4 ? 4 : 2;
    v4i held_of[AHEAD][LOADS];
    auto fetch_step = [&](int s, auto slot) {
        v4i(&held)[LOADS] = held_of[slot];
        const int k0 = first + s * BK;
        const unsigned some = s < steps ? ~0u : 0u;        // (behind the last step all lanes read one place, which costs less)
        const int8_t *const w0 = a.w + n0 * a.ldw, *const w1 = (GATED ? a.w2 : a.w) + n0 * a.ldw, *const x0 = a.x + m0 * a.ldx;
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const bool up = GATED && (((j * NW + wave) * ROWS) & 32);
            held[j] = *(const v4i_any *)((up ? w1 : w0) + ((off_w[j] + (unsigned)min(k0, a.K - 16 - 16 * piece_w[j])) & some));
        }
#pragma unroll
        for (int j = 0; j < LX; ++j) held[LW + j] = *(const v4i_any *)(x0 + ((off_x[j] + (unsigned)min(k0, a.K - 16 - 16 * piece_x[j])) & some));
    };
    auto put_step = [&](int s, auto slot) {
        v4i(&held)[LOADS] = held_of[slot];
        uint8_t *const to = lds + (s % STAGES) * STAGE + wave * 1024 + lane * 16;
        const int left = a.K - first - s * BK;
        if (left < BK) {
#pragma unroll
            for (int j = 0; j < LX; ++j) held[LW + j] = last_of(held[LW + j], left - 16 * piece_x[j]);
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) *(v4i *)(to + (j < LW ? j * NW * 1024 : BN * BK + (j - LW) * NW * 1024)) = held[j];
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

    // The order of a slice's products, the reads of the next one's fragments and the copies among them: reads under the first half of the products, copies under
    // the second, so that neither queue stops the wave between two products.
    auto order = [&](auto copies) {
        constexpr int M = TN * TM, R = TN + TM, H = M / 2, C = copies;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            const int reads = m < H ? R * (m + 1) / H - R * m / H : 0, cs = m < H ? 0 : C * (m - H + 1) / (M - H) - C * (m - H) / (M - H);
            if (reads == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (reads == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            if (reads >= 3) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
            if (cs == 1) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            if (cs == 2) __builtin_amdgcn_sched_group_barrier(0x010, 2, 0);
            if (cs >= 3) __builtin_amdgcn_sched_group_barrier(0x010, 4, 0);
        }
    };
    typedef std::integral_constant<int, 0> None;
    typedef std::integral_constant<int, LOADS / 2> Half;
    typedef std::integral_constant<int, LOADS> All;
    if (DIRECT) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s)
            if (s < STAGES - 1) copy_part(s, None{}, All{});
            else copy_part(s, None{}, Half{});
        FFN_WAIT_VMCNT((STAGES - 2) * LOADS + LOADS / 2);
    } else {
        times(std::integral_constant<int, AHEAD>{}, [&](auto u) { fetch_step(u, u); });
        put_step(0, None{});
        fetch_step(AHEAD, None{});
        FFN_WAIT_LGKM();
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_slice(0, 0, 0);
    // A stage's last slice is multiplied behind the barrier: its fragments have left LDS in front of it, so the stage is free for the copies of the step STAGES
    // further on (half of them there, half in the next step's first slice), and the first fragments of the next step come in under those products.
    auto one_step = [&](int s, auto next, auto more) {     // next: the slot of step s + 1; more: whether to load into it what comes AHEAD steps later
#pragma unroll
        for (int kk = 0; kk < SLICES - 1; ++kk) {
            read_slice(s % STAGES, kk + 1, (kk + 1) & 1);
            if (DIRECT && kk == 0) copy_part(s + STAGES - 1, Half{}, All{});
            multiply(kk & 1);
            if (DIRECT && kk == 0) order(std::integral_constant<int, LOADS - LOADS / 2>{});
            else order(None{});
        }
        if (DIRECT) FFN_WAIT_VMCNT((STAGES - 2) * LOADS);              // (the stages behind the next one are still in flight)
        else put_step(s + 1, next);
        FFN_WAIT_LGKM();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read_slice((s + 1) % STAGES, 0, 0);
        if (DIRECT) copy_part(s + STAGES, None{}, Half{});
        else if (more) fetch_step(s + 1 + AHEAD, next);
        multiply(1);
        if (DIRECT) order(Half{});
    };
    int s = 0;
    for (; s + AHEAD <= steps; s += AHEAD)
        times(std::integral_constant<int, AHEAD>{}, [&](auto u) { one_step(s + u, std::integral_constant<int, (u + 1) % AHEAD>{}, std::true_type{}); });
    times(std::integral_constant<int, AHEAD - 1>{}, [&](auto u) {
        if (s + u < steps) one_step(s + u, std::integral_constant<int, u + 1>{}, std::false_type{});
    });
    FFN_WAIT_VMCNT(0);
    drain(acc);

    if (ta.splits > 1) {
        // The partial sums are written through to memory and read past the caches (16: a scope of the whole chip), so they are coherent between the XCDs' L2
        // caches; a store has reached memory when the wave's counter of outstanding operations says so.  No workgroup waits for another.
        constexpr unsigned UNIT = NW * 64 * TN * TM * 64;
        const __amdgpu_buffer_rsrc_t rs_part = __builtin_amdgcn_make_buffer_rsrc((void *)ta.part, 0, 0x7fffffff, 0x20000);
        const unsigned mine = (unsigned)unit * UNIT + threadIdx.x * 16;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    __builtin_amdgcn_raw_buffer_store_b128(v4i{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]}, rs_part,
                                                           mine + ((i * TM + j) * 4 + e) * (NW * 1024), 0, 16);
        asm volatile("" ::: "memory");
        FFN_WAIT_VMCNT(0);
        __syncthreads();                                   // every wave's sums are in memory, and LDS is free
        if (threadIdx.x == 0) {
            const bool last = atomicAdd(ta.counters + slot, 1u) == (unsigned)ta.splits - 1;
            if (last) ta.counters[slot] = 0;               // all have arrived: ready for the next call
            *(int *)lds = last;
        }
        __syncthreads();
        if (!*(const int *)lds) return;
        constexpr int AT_ONCE = TN * TM <= 2 ? 4 : 1;      // ranges whose sums are on their way together
        for (int o = 1; o < ta.splits; o += AT_ONCE) {
            v4i t[AT_ONCE][TN * TM * 4];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                if (o + u >= ta.splits) continue;
                const int other = range + o + u < ta.splits ? range + o + u : range + o + u - ta.splits;
                const unsigned theirs = (unsigned)(slot * ta.splits + other) * UNIT + threadIdx.x * 16;
#pragma unroll
                for (int g = 0; g < TN * TM * 4; ++g) t[u][g] = __builtin_amdgcn_raw_buffer_load_b128(rs_part, theirs + g * (NW * 1024), 0, 16);
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                if (o + u >= ta.splits) continue;
#pragma unroll
                for (int g = 0; g < TN * TM * 4; ++g) {
                    v16i &c = acc[g / 4 / TM][g / 4 % TM];
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[4 * (g & 3) + e] += t[u][g][e];
                }
            }
        }
    }

    // ---- epilogue.  The sums go through LDS (as many of the tile's rows at a time as fit) into an order in which a thread has eight outputs n next to each
    // other of row after row: it reads their scales and biases once, a row's residual and y are read and written in whole lines, and the loads of several rows are in
    // flight together.  Row q's 16-byte piece c lies at c ^ (q & 15).
    constexpr int OUT = GATED ? BN / 2 : BN, TPR = OUT / 8, PASS = NW * 64 / TPR;           // outputs, threads a row; rows a pass
    constexpr int FIT = STAGES * STAGE / (WM * 32 * BN * 4), JR = FIT >= TM ? TM : FIT >= 2 && TM % 2 == 0 ? 2 : 1, ROWS_R = WM * JR * 32;
    static_assert(FIT >= 1 && ROWS_R % (PASS * 2) == 0 && TM <= 4, "whole passes, at most four dumps");
    const int o = 8 * (threadIdx.x % TPR), q0 = threadIdx.x / TPR, n = n0 + o;
    const int c0 = (GATED ? (o >> 5) * 64 + (o & 31) : o) >> 2;                             // first piece of the thread's sums
    const bool some = n < a.N, all = n + 8 <= a.N;
    float s1[8] = {}, b1[8] = {}, s2[8] = {}, b2[8] = {};
    if (some) {
        load_column(a.ws, n, a.N, s1);
        if (a.bias) load_column(a.bias, n, a.N, b1);
        if (GATED) {
            load_column(a.ws2, n, a.N, s2);
            if (a.bias2) load_column(a.bias2, n, a.N, b2);
        }
    }
    auto barrier = [&]() {
        FFN_WAIT_LGKM();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // P rows of a thread at a time; the residual of the next ones is on its way
    const bool with_res = !GATED && a.res;
    auto dump = [&](auto j0) {
#pragma unroll
        for (int j = 0; j < JR; ++j)
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                const int q = (wm * JR + j) * 32 + r, c = (wn * TN + i) * 8 + 4 * half;
                const v16i &t = acc[i][j0 + j];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *(v4i *)(lds + q * (BN * 4) + (((c + e) ^ (q & 15)) << 4)) = v4i{t[4 * e], t[4 * e + 1], t[4 * e + 2], t[4 * e + 3]};
            }
    };
    auto finish = [&](auto dt) {
        constexpr int DT = dt, P = 2, TURNS = ROWS_R / PASS / P, ALL_TURNS = TM / JR * TURNS, DEPTH = ALL_TURNS % 2 ? 1 : 2, ITEM = DT == kF32 ? 4 : 2;
        // row q0 + (a number that is the same for all threads) of the tile
        static_assert(32 % PASS == 0 && P * PASS % 16 == 0, "a pass stays in a group's 32 rows, a turn's rows start at a multiple of 16");
        auto above = [&](int turn, int p) {
            const int q = ((turn % TURNS) * P + p) * PASS;
            return (q / (JR * 32) * TM + turn / TURNS * JR) * 32 + q % (JR * 32);
        };
        const int last = some ? a.M - m0 - q0 : 0;                                          // rows from the thread's first one on
        const float *const xs0 = a.xs + m0 + q0;
        const uint8_t *const res0 = (const uint8_t *)a.res + ((m0 + q0) * a.ldr + n) * ITEM;
        uint8_t *const y0 = (uint8_t *)a.y + ((m0 + q0) * a.ldy + n) * ITEM;
        Eight<DT> ahead[DEPTH][P] = {};
        float xs_ahead[DEPTH][P] = {};
        auto fetch = [&](int turn, int to) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int u = above(turn, p);
                if (u < last) {
                    xs_ahead[to][p] = xs0[u];
                    if (with_res) ahead[to][p] = all ? load_eight<DT>(res0 + u * a.ldr * ITEM, 0) : load_up_to_eight<DT>(res0 + u * a.ldr * ITEM, a.N - n);
                }
            }
        };
        auto one_turn = [&](int turn, auto slot) {
            if (turn && turn % TURNS == 0) {
                barrier();
                if (JR < TM && turn == TURNS) dump(std::integral_constant<int, (JR < TM ? JR : 0)>{});
                if (2 * JR < TM && turn == 2 * TURNS) dump(std::integral_constant<int, (2 * JR < TM ? 2 * JR : 0)>{});
                if (3 * JR < TM && turn == 3 * TURNS) dump(std::integral_constant<int, (3 * JR < TM ? 3 * JR : 0)>{});
                barrier();
            }
            const uint8_t *const from = lds + ((turn % TURNS) * P * PASS + q0) * (BN * 4);
            Eight<DT> res[P];
            float v[P * 8], xs[P];
            v4i t[P][GATED ? 4 : 2];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                res[p] = ahead[slot][p];
                xs[p] = xs_ahead[slot][p];
#pragma unroll
                for (int e = 0; e < (GATED ? 4 : 2); ++e)
                    t[p][e] = *(const v4i *)(from + p * PASS * (BN * 4) + (((c0 + (e & 1) + (e & 2) * 4) ^ ((q0 + p * PASS) & 15)) << 4));
            }
            if (turn + DEPTH < ALL_TURNS) fetch(turn + DEPTH, slot);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * p + e] = (float)t[p][e >> 2][e & 3] * xs[p] * s1[e] + b1[e];
            activate_all(v, a.act, DT);
            if (GATED) {
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * p + e] *= (float)t[p][GATED ? 2 + (e >> 2) : 0][e & 3] * xs[p] * s2[e] + b2[e];
            }
            if (with_res) {
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * p + e] += value_of<DT>(res[p], e);
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int u = above(turn, p);
                float out[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e] = v[8 * p + e];
                if (u < last) {
                    uint8_t *const at = y0 + u * a.ldy * ITEM;
                    if (all) {
                        store_eight<DT>(at, 0, out);
                    } else {
#pragma unroll
                        for (int e = 0; e < 7; ++e)
                            if (n + e < a.N) store_number(at, e, DT, out[e]);
                    }
                }
            }
        };
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) fetch(k, k);
        barrier();
        dump(std::integral_constant<int, 0>{});
        barrier();
#pragma unroll 1
        for (int turn = 0; turn < ALL_TURNS; turn += DEPTH) {
            one_turn(turn, std::integral_constant<int, 0>{});
            if constexpr (DEPTH == 2) one_turn(turn + 1, std::integral_constant<int, DEPTH - 1>{});
        }
    };
    if (a.dtype == kBf16) finish(std::integral_constant<int, kBf16>{});
    else if (a.dtype == kF16) finish(std::integral_constant<int, kF16>{});
    else finish(std::integral_constant<int, kF32>{});
#endif
}

// Rows and weights that start at multiples of 16 bytes, with whole 16-byte pieces of k, are copied without a stop in registers
static bool direct(const LinearArgs &a)
{
    const uintptr_t at = (uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.w2;
    return (at & 15) == 0 && ((a.ldx | a.ldw | a.K) & 15) == 0;
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES, bool GATED, bool DIRECT>
static hipError_t launch_one(const LinearArgs &a, int splits, hipStream_t st)
{
    constexpr int BN = 32 * TN * WN / (GATED ? 2 : 1), BM = 32 * TM * WM, LDS = 32 * (TN * WN + TM * WM) * BK * STAGES;
    TiledArgs t;
    t.l = a;
    t.tiles_n = (a.N + BN - 1) / BN;
    t.tiles_m = (a.M + BM - 1) / BM;
    const int steps = (a.K + BK - 1) / BK;
    t.steps_per = (steps + splits - 1) / splits;
    t.splits = (steps + t.steps_per - 1) / t.steps_per;    // (no range without a step)
    t.counters = (unsigned *)a.workspace;
    t.part = (int32_t *)((uint8_t *)a.workspace + kSplitCounterBytes);
    const long long units = (long long)t.tiles_n * t.tiles_m * t.splits, per = (units + 7) / 8;
    t.per_xcd = (int)per;
    auto *const k = linear_tiled_kernel<TN, TM, WN, WM, BK, STAGES, GATED, DIRECT>;
    if (LDS > 65536)
        if (hipError_t e = allow_large_lds((const void *)k)) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)(per * 8)), dim3(WN * WM * 64), LDS, st, t);
    return hipGetLastError();
}

template <int TN, int TM, int WN, int WM, int BK, int STAGES>
static hipError_t launch_tiles(const LinearArgs &a, int splits, hipStream_t st)
{
    if (direct(a))
        return a.w2 ? launch_one<TN, TM, WN, WM, BK, STAGES, true, true>(a, splits, st) : launch_one<TN, TM, WN, WM, BK, STAGES, false, true>(a, splits, st);
    return a.w2 ? launch_one<TN, TM, WN, WM, BK, 2, true, false>(a, splits, st) : launch_one<TN, TM, WN, WM, BK, 2, false, false>(a, splits, st);
}

// (the cases in the order of kTiles)
hipError_t launch_tiled_linear(const LinearArgs &a, const TilePlan &p, hipStream_t st)
{
    static_assert(kTileKinds == 6 && kSplitCounterBytes == kWsCounterBytes, "a case a tile; counters as in the other workspaces");
    switch (p.tile) {
    case 0: return launch_tiles<2, 4, 4, 2, 128, 2>(a, p.splits, st);
    case 1: return launch_tiles<2, 2, 4, 2, 128, 3>(a, p.splits, st);
    case 2: return launch_tiles<2, 2, 2, 2, 128, 2>(a, p.splits, st);
    case 3: return launch_tiles<2, 2, 2, 2, 128, 4>(a, p.splits, st);
    case 4: return launch_tiles<2, 1, 2, 2, 128, 3>(a, p.splits, st);
    default:                                               // (four waves where gate and up need not be in one: 24 x 256 -> 8192 3.6 us, by two waves 4.2)
        if (a.w2) return launch_tiles<2, 1, 1, 2, 128, 4>(a, p.splits, st);
        return direct(a) ? launch_one<1, 1, 2, 2, 128, 4, false, true>(a, p.splits, st) : launch_one<1, 1, 2, 2, 128, 2, false, false>(a, p.splits, st);
    }
}

}  // namespace icnn
