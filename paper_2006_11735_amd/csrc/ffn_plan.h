// How products of 8-bit rows are launched: by which kernel, in which tiles, in how many ranges of k.  Host arithmetic alone, so that it can be tested without a GPU.
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
inline float step_factor(const LinearArgs &a)
{
    const unsigned at = (unsigned)((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.w2) | (unsigned)(a.ldx | a.ldw);
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

}  // namespace icnn
