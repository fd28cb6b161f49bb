// Products of 8-bit rows and 4-bit weights, which have a scale for every `group` numbers of a row:
//   acc_g = sum over the numbers k of group g of x[m][k] w[n][k] (int32, exact), s = sum over g of ws[n][g] acc_g in float32,
//   v = s * xs[m] + bias[n], y[m][n] = act(v) + res[m][n] or, gated, act(v) * v2; rounded to the stream's type once.
// Weights are laid out once: a row is blocks of 32 numbers in 16 bytes, byte j with number j in its lower and number 16 + j in its upper half, so that a shift
// and a mask make two operands of the matrix instruction of them.  As they come they are 16 times the weights; the scales are taken over 16.
#include "ffn_s4.h"

namespace icnn {

// Wait states between the last products and their sums' first reader (see mfma_drain in conv_common.h)
__device__ __forceinline__ void drain(v4i &c, v4i &d) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(c), "+v"(d)); }

// One wave a tile of 16 x 16 outputs, operands straight from memory: any size, stride and alignment.
template <bool GATED, bool NARROW>
__global__ __launch_bounds__(256) void s4_plain_kernel(const LinearS4Args a, int tiles_n, long long tiles)
{
    const long long tile = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int m0 = (int)(tile / tiles_n) * 16, n0 = (int)(tile % tiles_n) * 16;
    const int8_t *const x = a.x + min(m0 + r, a.M - 1) * a.ldx;
    const long long at = min(n0 + r, a.N - 1) * a.ldw;
    const int blocks = (int)(a.ldw / kBlockBytes), step = NARROW ? 32 : 64;
    float sum[4] = {}, sum2[4] = {};
    // a matrix instruction's four parts of k, g, are the halves of two blocks; of groups of 32 the first or the second block's alone (NARROW)
    for (int i = 0; i < a.groups; ++i) {
        v4i acc[2] = {};
        for (int k0 = i * a.group; k0 < min((i + 1) * a.group, a.K); k0 += step) {
            const int b = (k0 >> 5) + (g >> 1);
            const bool none = b >= blocks || (NARROW && g > 1);
            const v4i xv = none ? v4i{} : load_k16(x, 32 * b + 16 * (g & 1), a.K);
            auto weights = [&](const uint8_t *w) {
                const v4i block = none ? v4i{} : *(const v4i *)(w + at + (long long)b * kBlockBytes);
                return g & 1 ? sixteen_of<true>(block) : sixteen_of<false>(block);
            };
            acc[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(weights(a.w), xv, acc[0], 0, 0, 0);
            if (GATED) acc[1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(weights(a.w2), xv, acc[1], 0, 0, 0);
        }
        drain(acc[0], acc[1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const long long s = (long long)min(n0 + 4 * g + e, a.N - 1) * a.groups + i;
            sum[e] += (float)acc[0][e] * group_scale(a.ws, s, a.scale_dtype);
            if (GATED) sum2[e] += (float)acc[1][e] * group_scale(a.ws2, s, a.scale_dtype);
        }
    }
    const int m = m0 + r;
    if (m < a.M) finish_four_s4<GATED>(a, sum, sum2, m, n0 + 4 * g);
}

template <bool GATED>
static void launch_plain(const LinearS4Args &a, hipStream_t st)
{
    const int tiles_n = (a.N + 15) / 16;
    const long long tiles = (long long)((a.M + 15) / 16) * tiles_n;
    const dim3 grid((unsigned)((tiles + 3) / 4));
    if (a.group == 32) hipLaunchKernelGGL((s4_plain_kernel<GATED, true>), grid, dim3(256), 0, st, a, tiles_n, tiles);
    else hipLaunchKernelGGL((s4_plain_kernel<GATED, false>), grid, dim3(256), 0, st, a, tiles_n, tiles);
}

hipError_t launch_linear_s4(const LinearS4Args &a, hipStream_t st)
{
    const S4Plan plan = plan_s4(a, linear_tuning());
    switch (plan.kernel) {
    case LinearKernel::tokens: return launch_tokens_s4(a, st);
    case LinearKernel::few: return launch_few_s4(a, st);
    case LinearKernel::tiled:
        switch (a.group) {
        case 32: return launch_tiled_s4_32(a, plan.tile, st);
        case 64: return launch_tiled_s4_64(a, plan.tile, st);
        case 128: return launch_tiled_s4_128(a, plan.tile, st);
        default: return launch_tiled_s4_256(a, plan.tile, st);
        }
    case LinearKernel::plain: break;
    }
    if (a.w2) launch_plain<true>(a, st);
    else launch_plain<false>(a, st);
    return hipGetLastError();
}

// w / scale to nearest, ties to even, in [-7, 7].  The quotient in float32 is on the side of a tie that the exact one is on, or on the tie itself: then the remainder says
// which of the three it is (half of a group's largest weight is 3.5 steps but for the rounding of its float32 scale; 38 % of such came out on the wrong side without).  The
// remainder is exact: below a scale of 1 it is taken of twice the numbers, since a half of a subnormal's last bit is none.
__device__ __forceinline__ int four_bits(float w, float scale)
{
    const float v = w / scale, below = floorf(v), up = scale < 1.f ? 2.f : 1.f;
    float t = rintf(v);
    if (v - below == 0.5f) {
        const float rest = __builtin_fmaf(-(v * up), scale, w * up);
        t = rest > 0.f ? below + 1.f : rest < 0.f ? below : t;
    }
    return (int)fminf(fmaxf(t, -7.f), 7.f);
}

// Weights to 4 bits: a thread has a block of 32 numbers, the group / 32 threads of a group are next to each other in a wave.  Bound by its loads, a number at a time, the lanes'
// 64 or 128 bytes apart: 16384 x 4096 in bfloat16 255 to 261 us, in float32 2450; a program does it once.
//   scale = max|w| / 7 of the group, rounded to its type; number = w / scale to nearest, ties to even, in [-7, 7]
__global__ __launch_bounds__(256) void quantize_s4_kernel(const QuantizeS4Args a, int per_row, long long units)
{
    const long long u = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long n = u / per_row;
    const int b = (int)(u - n * per_row), k0 = 32 * b, left = n < a.n ? min(32, a.k - k0) : 0;
    const uint8_t *const row = (const uint8_t *)a.w + n * a.ld * (a.dtype == kF32 ? 4 : 2);
    uint32_t most = 0;
    for (int i = 0; i < left; ++i) most = max(most, __builtin_bit_cast(uint32_t, load_number(row, k0 + i, a.dtype)) & 0x7fffffffu);
    for (int d = 1; d < a.group / 32; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    if (left <= 0 || u >= units) return;
    float scale = round_number(__builtin_bit_cast(float, most) / 7.f, a.scale_dtype);
    if (!(scale < __builtin_huge_valf())) scale = __builtin_nanf("");  // (a NaN or an infinity in the group, or a scale beyond its type)
    if (b % (a.group / 32) == 0) store_number(a.scale, n * ((a.k + a.group - 1) / a.group) + k0 / a.group, a.scale_dtype, scale);
    unsigned q[4] = {};
    for (int i = 0; i < left; ++i) {
        const int t = scale > 0.f ? four_bits(load_number(row, k0 + i, a.dtype), scale) : 0;
        const unsigned bits = (unsigned)(t & 15) << (8 * (i & 3) + (i & 16 ? 4 : 0));
        q[0] |= (i & 12) == 0 ? bits : 0;
        q[1] |= (i & 12) == 4 ? bits : 0;
        q[2] |= (i & 12) == 8 ? bits : 0;
        q[3] |= (i & 12) == 12 ? bits : 0;
    }
    *(v4i *)(a.packed + (n * ((a.k + 31) / 32) + b) * kBlockBytes) = v4i{(int)q[0], (int)q[1], (int)q[2], (int)q[3]};
}

hipError_t launch_quantize_s4(const QuantizeS4Args &a, hipStream_t st)
{
    const int per_row = (a.k + a.group - 1) / a.group * (a.group / 32);        // whole groups: a row's threads do not share one with the next row's
    const long long units = (long long)a.n * per_row, blocks = (units + 255) / 256;
    hipLaunchKernelGGL(quantize_s4_kernel, dim3((unsigned)blocks), dim3(256), 0, st, a, per_row, units);
    return hipGetLastError();
}

}  // namespace icnn
