// How products of 8-bit rows are launched: by which kernel, in which tiles, in how many ranges of k, and which tile a workgroup has.  Arithmetic alone, the host's and a kernel's,
// so that it can be tested without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace icnn {

// A product of 8-bit rows and 8-bit weights, or the two of a gated layer (see ffn_linear.hip)
struct LinearArgs {
    const int8_t *x, *w, *w2;       // w2 null: one product.  Else y = act(first) * second
    const float *xs, *ws, *ws2, *bias, *bias2;
    const void *res;
    void *y;
    void *workspace;                // null: k stays whole
    long long ldx, ldw, ldr, ldy;
    int M, N, K;
    int act, dtype;
};

// What icnn_set_tuning has set of "ff_kernel" and "ff_split"
struct LinearTuning {
    int kernel, split;
};

// A launch holds fewer than 2^32 threads
constexpr bool fits_launch(long long groups, int threads) { return groups <= 0xffffffffLL / threads; }

// How much longer a step along k is where rows go through registers: with k whole 64 x 5456 -> 2048 (rows at multiples of 16) 15.2 us,
// 5464 (of 8) 15.8, 5461 19.8; 4096 x 2048 -> 8192 in 256 x 256 tiles 87 us, 2047 112
constexpr float kStepFactors[] = {1.f, 1.2f, 1.7f};         // rows at multiples of 16 bytes, of 4, anywhere
inline float step_factor(const LinearArgs &a, long long expert_stride = 0)
{
    const unsigned at = (unsigned)((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.w2) | (unsigned)(a.ldx | a.ldw | expert_stride);
    return kStepFactors[at & 3 ? 2 : (at | (unsigned)a.K) & 15 ? 1 : 0];
}

// (eight rows: 4096 -> 16384 15.4 us, by the kernel for few rows 16.1; 8192 -> 8192 16.1 and 14.7)
inline bool tokens_linear_takes(const LinearArgs &a) { return a.M <= 4 && a.K >= 16 && a.K <= 32768; }

// The kernel for few rows: waves of a workgroup, bytes of a weight row that a wave takes a turn
constexpr int kFewWaves = 4, kFewTurn = 256;
// A tile's rows within 2 GiB of its first; k is at least a piece
inline bool few_linear_takes(const LinearArgs &a) { return a.M <= 64 && a.K >= 16 && a.ldw <= (1 << 26); }

// Measured: a start, so much a megabyte of weights and so much for each time that the chip is filled with workgroups (each reads all rows; gated ones do it for
// twice the weights), or a turn of a wave where few workgroups are on the chip (8 rows, 4096 -> 16384: 16.5 us, 8192 -> 8192: 14.7, gated 4096 -> 16384: 26.6; 16 rows,
// 4096 -> 4096: 7.6, 1024 -> 16384: 9.1; 32 rows, 16384 -> 4096: 23, 4096 -> 16384: 27.8; 64 rows, 4096 -> 4096: 14.4, 16384 -> 512: 35)
inline float few_linear_us(const LinearArgs &a, float step)
{
    const float mb = (a.w2 ? 2.f : 1.f) * (float)a.N * (float)a.K * 1e-6f, turns = (float)((a.K + kFewWaves * kFewTurn - 1) / (kFewWaves * kFewTurn));
    const float fills = (a.w2 ? 0.5f : 1.f) * (float)a.N / 4096.f;
    const float flow = a.M <= 8 ? 3.f + 0.165f * mb + 0.35f * fills : a.M <= 16 ? 3.f + 0.19f * mb + 0.9f * fills : a.M <= 32 ? 3.f + 0.21f * mb + 2.2f * fills : 6.5f + 0.47f * mb;
    const float chain = 3.f + turns * (a.M <= 16 ? 0.8f : a.M <= 32 ? 0.85f : 2.f);
    // (loads at odd places hold up a compute unit's other ones: 8 and 16 rows, 5461 -> 5000: 17.9 and 23.3 us, 5461 -> 2048: 10 and 12.6)
    const float slow = step < 1.5f ? step : a.M <= 8 ? 2.f : a.M <= 16 ? 2.6f : 3.2f, slow_chain = step < 1.5f ? step : 0.7f * slow;
    const float by_flow = slow * (flow - 3.f), by_chain = slow_chain * (chain - 3.f);
    return 3.f + (by_flow > by_chain ? by_flow : by_chain);
}

constexpr size_t kSplitCounterBytes = 4096;        // of a workspace's start: a counter a tile

// Offsets in a tile's rows within 2 GiB; k is at least a piece
inline bool tiled_linear_takes(const LinearArgs &a) { return a.K >= 16 && a.ldx <= (1 << 22) && a.ldw <= (1 << 22); }

// Which tile, and in how many ranges of k.  A tile's time is a part that does not depend on k (start, epilogue) and one for each 128 bytes of k; tiles beyond what
// the 256 compute units hold at a time wait for another turn.  Measured in us: {rows, weight rows, held at a time, fixed, a step with few tiles on the chip, a
// step with all}.
struct TileCost {
    int m, n, held;
    float fixed, few, all;
};
constexpr TileCost kTiles[] = {
    {256, 256, 256, 14.f, 1.15f, 1.75f},    // 4096 x 4096 -> 4096: 72 us (the next one: 78)
    {128, 256, 256, 8.f, 0.55f, 1.f},       // gated 512 x 4096 -> 8192: 40 us (the one before 59, the next one 45)
    {128, 128, 512, 6.f, 0.58f, 1.25f},     // two workgroups on a compute unit
    {128, 128, 256, 8.5f, 0.48f, 0.58f},    // ... one, with four stages instead of two: 1024 x 4096 -> 4096: 25 us (the one before 34, the next one 27)
    {64, 128, 512, 4.f, 0.29f, 0.75f},      // gated 77 x 2048 -> 5461: 10.1 us (the next one 11.1), -> 5456: 9.3 (10.2)
    {64, 64, 512, 3.f, 0.22f, 0.46f},       // 128 x 4096 -> 4096: 9.2 us (the one before 10.8), 512 x 4096 -> 4096: 15.9 us (15.7); gated, by half the waves, 1.5 us more
};
constexpr int kTileKinds = sizeof(kTiles) / sizeof(kTiles[0]);
constexpr int kMostSplits = 16, kSplitTiles = (int)(kSplitCounterBytes / sizeof(unsigned));
// us: the sums' way through memory and back, so much more for each range that one workgroup adds, and for each 64 x 64 sums that take it (64 x 16384 -> 512 in 64 x 64
// tiles: whole 28.3 us, in 2, 4, 8, 16 ranges 17.5, 12.0, 10.5, 12.5; 512 x 4096 -> 4096 in two ranges of 64 x 128 tiles 23.6, whole 15.7)
constexpr float kExchange = 0.5f, kExchangeRange = 0.55f, kExchangeSums = 0.006f;

struct TilePlan {
    int tile, splits;
    float us;
};

inline TilePlan plan_tiles(const LinearArgs &a, const LinearTuning &tuning, float step, bool may_split)
{
    TilePlan best = {0, 1, 0.f};
    const int steps = (a.K + 127) / 128;
    for (int c = 0; c < kTileKinds; ++c) {
        if (tuning.kernel >= 4 && c != tuning.kernel - 4) continue;
        const TileCost &t = kTiles[c];
        const float tiles = (float)((a.M + t.m - 1) / t.m) * (float)(((a.w2 ? 2ll : 1ll) * a.N + t.n - 1) / t.n);
        for (int s = 1; s <= kMostSplits; ++s) {
            if (s > 1 && (!may_split || tiles > (float)kSplitTiles || tiles * (float)s > (float)t.held || 2 * s > steps)) break;
            // (one workgroup on each unit: all of the chip, or, of the tiles that two share a unit, a quarter of the way there; through registers less of it, and
            // all where any unit has two: 384 x 5461 -> 2048 in 64 x 64 tiles 0.36 us a step, 1000 x 5461 -> 2048 0.73)
            const float units = tiles * (float)s, turns = __builtin_ceilf(units / (float)t.held), on = units < (float)t.held ? units / 256.f : (float)t.held / 256.f;
            const float full = t.held == 256 ? on : step > 1.f ? (on > 1.f ? 1.f : 0.15f * on) : on < 1.f ? 0.25f * on : 0.25f + 0.75f * (on - 1.f), more = c == kTileKinds - 1 && a.w2 ? 1.5f : 0.f;
            const float us = turns * (t.fixed + more + (float)((steps + s - 1) / s) * step * (t.few + (t.all - t.few) * full)) + (s > 1 ? kExchange + kExchangeRange * (float)s + kExchangeSums * units * (float)(t.m * t.n / 4096) : 0.f);
            if (tuning.split ? s == 1 || s <= tuning.split : best.us == 0.f || us < best.us) best = {c, s, us};
        }
    }
    return best;
}

// (no less than the weights take from memory: 8 x 4096 -> 16384 18.8 us, 8 x 8192 -> 8192, in two ranges of k, 21.1, gated 16 x 4096 -> 16384 31.7, which the
// kernel for few rows has in 28.3)
inline float tiled_linear_us(const LinearArgs &a, const TilePlan &p)
{
    const float flow = 3.f + 0.205f * (a.w2 ? 2.f : 1.f) * (float)a.N * (float)a.K * 1e-6f + (p.splits > 1 ? 3.f : 0.f);
    return p.us > flow ? p.us : flow;
}

// Up to four rows go token by token (1 x 16384 -> 4096: 12.4 us, by the kernel for few rows 17.6; 4 rows: 14.1 and 16.4), the others where they take least by what
// has been measured; what none of those takes (k below 16, rows gigabytes apart) by the plain kernel.
enum class LinearKernel { plain, tokens, few, tiled };
struct LinearPlan {
    LinearKernel kernel;
    TilePlan tiles;                // of LinearKernel::tiled
};

inline LinearPlan plan_linear(const LinearArgs &a, const LinearTuning &tuning, float step, bool may_split)
{
    const int force = tuning.kernel;
    const bool few = few_linear_takes(a), tiled = tiled_linear_takes(a);
    LinearPlan p = {LinearKernel::plain, {0, 1, 0.f}};
    if (tokens_linear_takes(a) && (force == 0 || force == 2)) {
        p.kernel = LinearKernel::tokens;
        return p;
    }
    if (tiled) p.tiles = plan_tiles(a, tuning, step, may_split);
    if (few && (force == 3 || (force == 0 && (!tiled || few_linear_us(a, step) < tiled_linear_us(a, p.tiles))))) p.kernel = LinearKernel::few;
    else if (tiled && (force == 0 || force >= 4)) p.kernel = LinearKernel::tiled;
    return p;
}

// What a launch does: the plan for its operands' addresses, in a workspace if there is one
inline LinearPlan plan_launch(const LinearArgs &a, const LinearTuning &tuning) { return plan_linear(a, tuning, step_factor(a), a.workspace != nullptr); }

// Bytes of the workspace that a plan uses
inline size_t plan_workspace(const LinearArgs &a, const LinearPlan &p)
{
    if (p.kernel != LinearKernel::tiled || p.tiles.splits == 1) return 0;
    const TileCost &t = kTiles[p.tiles.tile];
    const size_t tiles = (size_t)((a.M + t.m - 1) / t.m) * (size_t)(((a.w2 ? 2ll : 1ll) * a.N + t.n - 1) / t.n);
    return kSplitCounterBytes + tiles * (size_t)p.tiles.splits * (size_t)(t.m * t.n) * 4;
}

// A product whose outputs one launch might not hold goes in several: ranges of outputs n and, within, of rows.  As many as here fit by any kernel, on any rows and
// weights: 16 x 16 outputs a wave (the plain kernel), 64 x 32 (the smallest gated tile) or 64 x 64 by at most 256 threads, one output by at most 512 (single tokens).
constexpr long long kMostColumns = 1 << 22, kMostOutputs = 1ll << 33;
static_assert(fits_launch(kMostOutputs / 1024 + 1, 256) && fits_launch(kMostOutputs / 2048 + 8, 256) && fits_launch(kMostColumns, 512), "any kernel's launch");

inline long long rows_of_a_range(const LinearArgs &a)
{
    const long long columns = a.N < kMostColumns ? (a.N + 63ll) / 64 * 64 : kMostColumns;
    return kMostOutputs / columns / 256 * 256;
}

inline bool one_range(const LinearArgs &a) { return a.N <= kMostColumns && a.M <= rows_of_a_range(a); }

// fn of every range's operands, until it returns something.  `item`: bytes of an element of y.  Ranges of a larger product do not split k (they fill the chip; the last
// ones need not).
template <class F>
inline auto each_range(const LinearArgs &a, int item, F &&fn) -> decltype(fn(a))
{
    if (one_range(a)) return fn(a);
    const long long rows = rows_of_a_range(a);
    for (long long n = 0; n < a.N; n += kMostColumns)
        for (long long m = 0; m < a.M; m += rows) {
            LinearArgs b = a;
            b.M = (int)(a.M - m < rows ? a.M - m : rows);
            b.N = (int)(a.N - n < kMostColumns ? a.N - n : kMostColumns);
            b.x += m * a.ldx;
            b.xs += m;
            b.w += n * a.ldw;
            b.ws += n;
            if (a.bias) b.bias += n;
            if (a.w2) {
                b.w2 += n * a.ldw;
                b.ws2 += n;
            }
            if (a.bias2) b.bias2 += n;
            if (a.res) b.res = (const int8_t *)a.res + (m * a.ldr + n) * item;
            b.y = (int8_t *)a.y + (m * a.ldy + n) * item;
            b.workspace = nullptr;
            if (auto e = fn(b)) return e;
        }
    return {};
}

// Bytes that a caller is asked for, who may put the operands anywhere afterwards: the most that plan_launch comes to at any addresses.  They can but raise the
// step's factor above that of the strides and k, which `a` has here with operands at multiples of 16.
inline size_t linear_workspace(const LinearArgs &a, const LinearTuning &tuning)
{
    if (!one_range(a)) return 0;
    size_t most = 0;
    for (float step : kStepFactors) {
        if (step < step_factor(a)) continue;
        const size_t bytes = plan_workspace(a, plan_linear(a, tuning, step, true));
        most = bytes > most ? bytes : most;
    }
    return most;
}

// Products whose rows lie in the order of their experts (see ffn_grouped.hip): `l` has the first expert's weights, scales and biases, M is the number of positions
struct GroupedArgs {
    LinearArgs l;
    const int32_t *index;          // x's row of a position; null: the position itself
    const int32_t *offsets;        // expert e's positions: offsets[e] .. offsets[e + 1] - 1
    long long x_rows, expert_stride;
    int experts;
};

// Groups of `rows` positions of one expert each: as many as there can be, whatever the experts' shares are
inline long long grouped_slots(long long positions, int experts, int rows)
{
    return positions / rows + (positions < experts ? positions : experts);
}

// Operands' offsets in a tile within 2 GiB: rows of an index lie anywhere in x.  (Beyond, the kernel for few rows has them: 16384 positions of 8 experts, 8192 -> 4096, with an x of
// 260000 rows 558 us, of 300000 4580.)
inline bool grouped_rows_near(const GroupedArgs &a) { return a.index ? a.l.ldx <= (0x7ff00000ll / (a.x_rows > 0 ? a.x_rows : 1)) : a.l.ldx <= (1 << 22); }
inline bool grouped_tiled_takes(const GroupedArgs &a) { return a.l.K >= 16 && a.l.ldw <= (1 << 22) && grouped_rows_near(a); }
inline bool grouped_few_takes(const GroupedArgs &a) { return a.l.K >= 16 && a.l.ldw <= (1 << 26); }
inline bool grouped_tokens_takes(const GroupedArgs &a) { return a.l.K >= 16 && a.l.K <= 32768 && a.l.M <= 64; }

// (beside the sizes of kTiles: tiles of 256 x 256 and smaller ones in one launch)
constexpr int kMixedTiles = kTileKinds;

struct GroupedPlan {
    LinearKernel kernel;
    int tile;                      // of LinearKernel::tiled: its place in kTiles, or kMixedTiles
    int rows;                      // of LinearKernel::few: positions a group, 16, 32 or 64
};

// The experts' shares are not known here: they are taken to be even over those that so many positions are expected to reach, E (1 - exp(-M / E)).
inline GroupedPlan plan_grouped(const GroupedArgs &a, const LinearTuning &tuning, float step)
{
    const int force = tuning.kernel;
    const float positions = (float)a.l.M, experts = (float)a.experts, reached = experts * (1.f - __builtin_expf(-positions / experts)), share = positions / reached;
    GroupedPlan p = {LinearKernel::plain, 0, 16};
    // Position by position an expert's weights are read for each (8 positions of 8 experts, 1024 -> 2048: 4.8 us, by the kernel for few rows 5.8; 32 of 8: 8.8 and 6.7)
    if (grouped_tokens_takes(a) && (force == 2 || (force == 0 && share <= 1.6f && a.l.M <= 16))) {
        p.kernel = LinearKernel::tokens;
        return p;
    }
    // The kernel for few rows: a start, and a workgroup's own start and turns for each group and 16 outputs, more where groups are fuller, or a wave's turns one after the
    // other; rows at odd places take twice as long (64 positions of 64 experts: 1024 -> 2048 17.2 us, 4096 -> 1024 16.7, 2001 -> 1501 27.5, gated 32, 32 and 46; 256 of 64: 25,
    // 27 and 45; 32 of 8: 6.7, 9.1 and 11; 128 of 8: 12, 16 and 23)
    const bool few = grouped_few_takes(a), tiled = grouped_tiled_takes(a);
    const float turns_few = (float)((a.l.K + kFewWaves * kFewTurn - 1) / (kFewWaves * kFewTurn)), groups_few = reached * (share / 16.f + 0.6f) * (float)((a.l.N + 15) / 16);
    const float flow = (a.l.w2 ? 2.f : 1.f) * (step < 1.5f ? 1.f : 2.f) * (0.0024f + 0.0012f * turns_few) * groups_few, chain = turns_few * (share > 8.f ? 2.5f : 1.2f);
    const float few_us = 4.f + (flow > chain ? flow : chain);
    if (few && (force == 3 || (force == 0 && !tiled))) {
        p.kernel = LinearKernel::few;
        p.rows = share <= 16.f ? 16 : share <= 32.f ? 32 : 64;
        return p;
    }
    if (!tiled || (force != 0 && force < 4)) return p;
    p.kernel = LinearKernel::tiled;
    // Of an expert's last group half is taken to be empty.  The way to a tile, by offsets and index, is 2.5 us more than that of a dense one.
    float best = 0.f;
    const float steps = (float)((a.l.K + 127) / 128), weight_rows = (float)((a.l.w2 ? 2ll : 1ll) * a.l.N);
    for (int c = 0; c <= kMixedTiles; ++c) {
        if (force >= 4 && c != force - 4) continue;
        const TileCost &t = kTiles[c < kTileKinds ? c : 0];
        const float tiles_n = __builtin_ceilf(weight_rows / (float)t.n);
        float us;
        if (c == kMixedTiles) {
            const TileCost &half = kTiles[1];
            const float big = t.fixed + steps * step * t.all, small = half.fixed + steps * step * half.all, all = reached * tiles_n * (share / (float)t.m * big + 0.5f * small) / 256.f;
            us = (all > big ? all : big) + 0.4f * small;
        } else {
            const float groups = share / (float)t.m + 0.5f, tiles = reached * (groups > 1.f ? groups : 1.f) * tiles_n;
            const float turns = __builtin_ceilf(tiles / (float)t.held), on = tiles < (float)t.held ? tiles / 256.f : (float)t.held / 256.f;
            const float full = t.held == 256 ? on : step > 1.f ? (on > 1.f ? 1.f : 0.15f * on) : on < 1.f ? 0.25f * on : 0.25f + 0.75f * (on - 1.f);
            us = turns * (t.fixed + steps * step * (t.few + (t.all - t.few) * full));
        }
        us += 2.5f;
        if (best == 0.f || us < best) {
            best = us;
            p.tile = c;
        }
    }
    if (few && force == 0 && few_us < best) {
        p.kernel = LinearKernel::few;
        p.rows = 16;
    }
    return p;
}

// What a launch does: the plan for its operands' addresses, every expert's
inline GroupedPlan plan_grouped_launch(const GroupedArgs &a, const LinearTuning &tuning) { return plan_grouped(a, tuning, step_factor(a.l, a.expert_stride)); }

// Groups of ROWS positions of one expert each: all of them (the last one of an expert may have fewer), or those with more than half of ROWS, or an expert's rest of up
// to half, and of those the ones of more than a quarter, or of up to a quarter of ROWS
enum Groups { kAll, kWholeOrMost, kRest, kHalf, kQuarter };

template <int ROWS, Groups KIND>
constexpr int groups_among(int positions)
{
    const int rest = positions % ROWS;
    if (KIND == kRest) return rest > 0 && rest <= ROWS / 2;
    if (KIND == kHalf) return rest > ROWS / 4 && rest <= ROWS / 2;
    if (KIND == kQuarter) return rest > 0 && rest <= ROWS / 4;
    return positions / ROWS + (KIND == kAll ? rest > 0 : rest > ROWS / 2);
}

// Tile `slot` of tiles_m x tiles_n: eight rows of tiles, column after column, so that what an XCD has at one time shares its weights and rows
constexpr void tile_at(int slot, int tiles_m, int tiles_n, int *tm, int *tn)
{
    const int rows = 8, panel = slot / (rows * tiles_n), in_panel = slot - panel * rows * tiles_n, left = tiles_m - panel * rows, high = left < rows ? left : rows;
    *tn = in_panel / high;
    *tm = panel * rows + in_panel - *tn * high;
}

// Tiles of several sizes in one launch: an expert's positions in groups of 256, what is left of them in one of 256 or, up to 128 or 64, of so many.  Where the tiles of
// 256 x 256 do not fill the chip's 256 compute units once more, those beyond the last time they do may be cut in two of 128 x 256 or in eight of 64 x 128, and so may the
// rests' tiles of 128 x 256 in four: whatever is expected to end soonest.  In hundredths of a tile's time half of it takes 56 and an eighth `eighth` (8192 -> 8192: 37 us of
// 163, 1024 -> 8192 12 of 33).  EIGHTHS: from 32 steps of k on (2048 rows, top 2 of 8, 4096 -> 4096 103 us without, 97 with; 4096, top 4 of 32, 2048 -> 2048 108 and 111), but
// not in gated layers, where a wave needs both layers' rows: 64 rows take 40 there (2048, top 4 of 32, 2048 -> 2048 107 and 113; 98 to 110 by now).
// (4096 rows, top 2 of 8, 8192 -> 4096: 316 us in tiles of one size, 304 in two, 289 in three; the latter 276 to 286 by now.)
constexpr int kMixedRows = 256, kMostCut = 1024;           // workgroups that cuts may add

// Workgroups of such a launch, a multiple of 8: a group's tiles, or twice as many of a rest's; what cuts add; up to 7 / 8 of a workgroup for each XCD and size
template <bool EIGHTHS>
constexpr long long mixed_blocks(long long positions, int experts, int tiles_n)
{
    const long long groups = positions / kMixedRows + (positions < experts ? positions : experts), rests = groups - positions / kMixedRows;
    return (((EIGHTHS ? groups + rests : groups) * tiles_n + (EIGHTHS ? kMostCut : 256)) / 8 + 4) * 8;
}

// What a workgroup of it has: of the groups of kind `from` the `slot`-th, `down` rows further on, and the n-th tile of its columns; rows 256, 128 or 64; 0: nothing
struct MixedTile {
    int rows, slot, n, down;
    Groups from;
};

// groups, rests, small: how many of kWholeOrMost, of kRest (kHalf with EIGHTHS) and of kQuarter there are.  tiles_n, tiles8_n: tiles of 256 and of 64 rows beside each other
template <bool EIGHTHS>
constexpr MixedTile mixed_tile(int groups, int rest_groups, int small_groups, int tiles_n, int tiles8_n, int steps, unsigned block)
{
    constexpr Groups REST = EIGHTHS ? kHalf : kRest;
    constexpr int ROWS = kMixedRows, PARTS = 8, HALF = 56;
    const int eighth = 22 + 120 / steps, whole = groups * tiles_n, rests = rest_groups * tiles_n, beyond = whole & 255, small = EIGHTHS ? small_groups * tiles8_n : 0;
    // Of the tiles beyond the last full turn `in2` are cut in halves or `in8` in eighths, of the rests' halves `in4` in quarters
    int in2 = 0, in8 = 0, in4 = 0, least = 0x7fffffff;
    auto option = [&](int h, int e, int r) {
        if (h + e * (PARTS - 1) + r * (PARTS / 2 - 1) > kMostCut) return;
        const int bigs = beyond - h - e, halves = rests + 2 * h - r, eighths = small + e * PARTS + r * (PARTS / 2), more = halves - (256 - bigs);
        const int first = bigs ? 100 : 0, then = halves ? (first > HALF ? first : HALF) + HALF * (((more > 0 ? more : 0) + 255) / 256) : first;
        const int all = (100 * bigs + HALF * halves + eighth * eighths) / 256 + (eighths ? eighth / 2 : 0), end = then > all ? then : all;
        if (end < least) {
            least = end;
            in2 = h;
            in8 = e;
            in4 = r;
        }
    };
    option(0, 0, 0);
    option(beyond, 0, 0);
    if (EIGHTHS) {
        option(0, beyond, 0);
        option(0, beyond, rests);
        option(beyond, 0, rests);
    }
    const int bigs = whole - in2 - in8, halves = rests + 2 * in2 - in4, eighths = small + in8 * PARTS + in4 * (PARTS / 2);
    const int x = (int)(block & 7), per_big = (bigs + 7) / 8, per_half = (halves + 7) / 8, per_eighth = (eighths + 7) / 8;
    const int i = (int)(block >> 3), i2 = i - per_big, i8 = i2 - per_half;
    MixedTile t = {0, 0, 0, 0, kWholeOrMost};
    if (i2 < 0) {
        const int unit = x * per_big + i;
        if (unit >= bigs) return t;
        tile_at(unit, groups, tiles_n, &t.slot, &t.n);
        t.rows = ROWS;
    } else if (i8 < 0) {
        const int unit = x * per_half + i2, of_rests = unit - 2 * in2;
        if (unit >= halves) return t;
        if (of_rests < 0) {
            tile_at(bigs + unit / 2, groups, tiles_n, &t.slot, &t.n);
            t.down = ROWS / 2 * (unit & 1);
        } else {
            t.slot = of_rests / tiles_n;
            t.n = of_rests - t.slot * tiles_n;
            t.from = REST;
        }
        t.rows = ROWS / 2;
    } else if (EIGHTHS) {
        const int unit = x * per_eighth + i8, of_rests = unit - in8 * PARTS, of_small = of_rests - in4 * (PARTS / 2);
        if (i8 >= per_eighth || unit >= eighths) return t;
        if (of_small < 0) {                                // 64 rows and half the columns of a tile
            const int part = of_rests < 0 ? unit % PARTS : of_rests % (PARTS / 2), tile = of_rests < 0 ? bigs + unit / PARTS : of_rests / (PARTS / 2);
            if (of_rests < 0) {
                tile_at(tile, groups, tiles_n, &t.slot, &t.n);
            } else {
                t.slot = tile / tiles_n;
                t.n = tile - t.slot * tiles_n;
                t.from = REST;
            }
            t.down = ROWS / 4 * (part / 2);
            t.n = 2 * t.n + part % 2;
        } else {
            t.slot = of_small / tiles8_n;
            t.n = of_small - t.slot * tiles8_n;
            t.from = kQuarter;
        }
        if (t.n < tiles8_n) t.rows = ROWS / 4;
    }
    return t;
}

// What one launch holds by any kernel: 16 x 16 outputs a wave
constexpr long long kMostTiles = 1 << 25;
inline bool grouped_fits(long long positions, int experts, int n) { return grouped_slots(positions, experts, 16) <= kMostTiles / ((n + 15ll) / 16); }
inline bool s4_fits(long long rows, int n) { return (rows + 15) / 16 <= kMostTiles / ((n + 15ll) / 16); }

// A product of 8-bit rows and 4-bit weights, or the two of a gated layer (see ffn_s4.hip)
struct LinearS4Args {
    const int8_t *x;
    const uint8_t *w, *w2;         // rows of `ldw` bytes, blocks of 32 numbers in 16; w2 null: one product
    const float *xs, *bias, *bias2;
    const void *ws, *ws2;          // a scale for each group of a row's numbers: [n][groups]
    const void *res;
    void *y;
    long long ldx, ldr, ldy, ldw;
    int M, N, K;
    int group, groups;             // numbers of a group (32, 64, 128 or 256), groups of a row
    int act, dtype, scale_dtype;
};

// Tiles of a product with 4-bit weights, one on a compute unit at a time: {rows, weight rows, us that do not depend on k, us for 128 numbers of k in groups of 32, of 64 and of
// 128 or 256}.  Measured with 8192 -> 8192: 1024 rows by the first 84 us (by the second 98), 512 by the second 50 (84), 64 by the third 18 (46), 24 by the fourth 13 (18), 400
// with 8192 -> 512 by the fourth 11.9 (16.7); in groups of 32 1024 rows 156 us by the first (177).  The fourth, with eight waves along k, is for products with one set of weights.
struct S4TileCost {
    int m, n;
    float fixed, step[3];
};
constexpr S4TileCost kS4Tiles[] = {{128, 256, 9.f, {2.3f, 1.5f, 1.17f}}, {128, 128, 9.f, {1.25f, 0.8f, 0.64f}}, {64, 32, 4.f, {0.28f, 0.23f, 0.21f}}, {32, 32, 4.f, {0.14f, 0.12f, 0.11f}}};
constexpr int kS4TileKinds = sizeof(kS4Tiles) / sizeof(kS4Tiles[0]), kS4TileThreads = 512;

struct S4Plan {
    LinearKernel kernel;
    int tile;                      // of LinearKernel::tiled: its place in kS4Tiles
};

// (All on operands that no cache holds.)  Up to four rows token by token (1 x 16384 -> 4096: 8.3 us, by the kernel for few rows 16), up to 16 by the kernel for few rows, up to 32 by that or in tiles by what has
// been measured (24 rows: 4096 -> 4096 7.7 us, in tiles 8.5, 8192 -> 8192 15.3 and 13.3; 32 rows, gated 4096 -> 16384: 33 and 26), the others in tiles; k below 16 and rows
// gigabytes apart by the plain kernel
inline S4Plan plan_s4(const LinearS4Args &a, const LinearTuning &tuning)
{
    const int force = tuning.kernel;
    if (a.M <= 4 && a.K >= 16 && a.K <= 32768 && (force == 0 || force == 2)) return {LinearKernel::tokens, 0};
    const bool few = a.M <= 32 && a.K >= 16, tiled = a.K >= 16 && a.ldx <= (1 << 22);
    if (few && (force == 3 || (force == 0 && (a.M <= 16 || !tiled)))) return {LinearKernel::few, 0};
    if (!tiled || (force != 0 && force < 4)) return {LinearKernel::plain, 0};
    const int steps = (a.K + 127) / 128, by_group = a.group == 32 ? 0 : a.group == 64 ? 1 : 2;
    S4Plan p = {LinearKernel::plain, 0};
    float best = 0.f;
    const int kinds = a.w2 ? 3 : kS4TileKinds, only = force < 4 ? -1 : force - 4 < kinds ? force - 4 : kinds - 1;
    for (int c = 0; c < kinds; ++c) {
        const S4TileCost &t = kS4Tiles[c];
        if (only >= 0 && c != only) continue;
        const bool wider = a.w2 && c == 2;                 // (the third one's weight rows are twice as many in a gated layer, for a third more time)
        const long long tiles = ((a.M + t.m - 1ll) / t.m) * (((a.w2 ? 2ll : 1ll) * a.N + (wider ? 2 : 1) * t.n - 1) / ((wider ? 2 : 1) * t.n));
        if (!fits_launch(tiles + 7, kS4TileThreads)) continue;             // (of half a billion rows the first tile's always does)
        const float us = __builtin_ceilf((float)tiles / 256.f) * (t.fixed + (wider ? 1.3f : 1.f) * (float)steps * t.step[by_group]);
        if (best == 0.f || us < best) {
            best = us;
            p = {LinearKernel::tiled, c};
        }
    }
    // The kernel for few rows: a start, and the weights' way (megabytes), which the rows at odd places hold up, or a wave's turns of 128 bytes one after the other.  Tiles take 3 us
    // more on such rows.  (32 rows, 2001 -> 5461: 9.1 us, in tiles 9.1, gated 16.7 and 12.3.)
    const bool odd = (((uintptr_t)a.x | (uintptr_t)a.ldx) & 3) != 0;
    const float mb = (a.w2 ? 2.f : 1.f) * (float)a.N * (float)a.ldw * 1e-6f, way = (odd ? 0.9f : 0.36f) * mb, chain = 1.7f * (float)a.ldw / 1024.f;
    const float few_us = 4.f + (a.group == 32 ? 1.35f : 1.f) * (way > chain ? way : chain);
    if (few && force == 0 && few_us < 1.1f * (best + (odd ? 3.f : 0.f))) p.kernel = LinearKernel::few;
    return p;
}

}  // namespace icnn
