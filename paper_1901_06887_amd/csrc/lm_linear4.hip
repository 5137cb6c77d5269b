// mt_linear4: rows of many tenants times their 4-bit matrices.
//
// y[i][n] = act(b[n] + sum_k W[n][k] x[i][k]).  The weights are the row operand of the 16x16x32 bf16 matrix instruction, 16 rows of x the
// column operand: every e2m1 value times its scale is a bf16 value, every bf16 row value is itself one, an 8-bit one with its scale too, and an fp32
// one is the sum of three; so the products are exact and the sums fp32.  Lane l of an operand holds output (or row) l % 16 and the 32 values of k
// block l / 16, which is how the weights lie in memory: one 16-byte load a lane is an operand, with one scale, converted in place.
#include "lm_device.h"

namespace mt {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct RowsF32 { };
struct RowsBf16 { };
struct RowsMx8 { };

// 32 values of k of a row (a lane's share of a k tile) as matrix operands.
template <typename X> struct Operand { static constexpr int kParts = 1; u32x4 v[1][4]; };
template <> struct Operand<RowsF32> { static constexpr int kParts = 3; u32x4 v[3][4]; };

// fp32 as three bf16 values whose sum it is: the upper halves of what is left.  An infinity or NaN is the first alone.
__device__ __forceinline__ void split3(float x, uint32_t (&part)[3])
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const bool special = (b & 0x7f800000u) == 0x7f800000u;
    part[0] = b & 0xffff0000u;
    const float r = x - __builtin_bit_cast(float, part[0]);
    part[1] = __builtin_bit_cast(uint32_t, r) & 0xffff0000u;
    const float q = r - __builtin_bit_cast(float, part[1]);
    part[2] = __builtin_bit_cast(uint32_t, q) & 0xffff0000u;
    if (special) { part[0] |= (b & 0xffffu) ? 0x400000u : 0u; part[1] = part[2] = 0; }
}

// A lane's 32 values from column `at` of a row of `width`; zeros past its end, and where the row does not exist.
__device__ __forceinline__ void load_operand(Operand<RowsBf16>& o, const Linear4Args& a, uint64_t row, uint32_t at, uint32_t width, bool there)
{
    const __bf16* p = (const __bf16*)a.x + row * a.x_stride + at;
    if (there && at + 32 <= width) {
#pragma unroll
        for (int j = 0; j < 4; ++j) o.v[0][j] = *(const Any<__bf16>::vec16*)(p + 8 * j);
        return;
    }
    const uint32_t n = there && at < width ? width - at : 0;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t k = 8 * j + 2 * i;
            const uint32_t lo = k < n ? ((const uint16_t*)p)[k] : 0, hi = k + 1 < n ? ((const uint16_t*)p)[k + 1] : 0;
            o.v[0][j][i] = lo | hi << 16;
        }
}
__device__ __forceinline__ void load_operand(Operand<RowsF32>& o, const Linear4Args& a, uint64_t row, uint32_t at, uint32_t width, bool there)
{
    const float* p = (const float*)a.x + row * a.x_stride + at;
    const uint32_t n = there && at < width ? (width - at < 32 ? width - at : 32) : 0;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        float f[8];
        if (n == 32) load8(p + 8 * j, f); else load_some(p + 8 * j, n > 8 * j ? n - 8 * j : 0, f);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            uint32_t lo[3], hi[3];
            split3(f[2 * i], lo); split3(f[2 * i + 1], hi);
#pragma unroll
            for (int q = 0; q < 3; ++q) o.v[q][j][i] = lo[q] >> 16 | hi[q];
        }
    }
}
__device__ __forceinline__ void load_operand(Operand<RowsMx8>& o, const Linear4Args& a, uint64_t row, uint32_t at, uint32_t width, bool there)
{
    const uint8_t* p = (const uint8_t*)a.x + row * a.x_stride + at;
    const uint32_t n = there && at < width ? (width - at < 32 ? width - at : 32) : 0;
    uint32_t w[8];
    if (n == 32) {
        const u32x4 w0 = *(const Any<uint8_t>::vec16*)p, w1 = *(const Any<uint8_t>::vec16*)(p + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[i] = w0[i]; w[4 + i] = w1[i]; }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            w[i] = 0;
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) if (4 * i + e < n) w[i] |= (uint32_t)p[4 * i + e] << (8 * e);
        }
    }
    const uint32_t sb = n ? a.x_scales[row * a.x_scales_stride + at / MT_MX_BLOCK] : 127;
    // 2^(sb - 127); the smallest is subnormal, the largest byte is NaN
    const float scale = __builtin_bit_cast(float, sb == 0xff ? 0x7fc00000u : sb ? sb << 23 : 0x00400000u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        o.v[0][i / 2][i % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
        o.v[0][i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
    }
}

// A lane's 32 weights, scaled, as operands of four matrix instructions.
__device__ __forceinline__ void weights_of(const u32x4& codes, uint32_t scale_byte, u32x4 (&w)[4])
{
    const float s = __builtin_bit_cast(float, scale_byte << 23);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        w[j][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], s, 0));
        w[j][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], s, 1));
        w[j][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], s, 2));
        w[j][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], s, 3));
    }
}

// NaN stays NaN in both.
__device__ __forceinline__ float activate4(float z, uint32_t act)
{
    if (act == MT_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (act == MT_ACT_GELU) return 0.5f * z * erfcf(-0.70710678f * z);
    return z;
}

__device__ __forceinline__ void store4(__bf16* p, const f32x4& v)
{
    *(Any<__bf16>::vec8*)p = Any<__bf16>::vec8{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}
__device__ __forceinline__ void store4(float* p, const f32x4& v) { *(Any<float>::vec16*)p = __builtin_bit_cast(u32x4, v); }

// WK waves share the k tiles of 16 outputs times 16 rows and add their sums up through LDS.
template <typename X, typename Y, int WK>
__global__ void __launch_bounds__(WK * 64) linear4_kernel(Linear4Args a)
{
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the group is the last one that starts at or before this workgroup
    const bool starts = lane < a.n_groups && a.groups[lane < a.n_groups ? lane : 0].wg_base <= blockIdx.x;
    const uint32_t gi = __builtin_amdgcn_readfirstlane(__popcll(__ballot(starts)) - 1);
    const Group4& g = a.groups[gi];
    const uint32_t N = g.N, K = g.K;
    const uint32_t n_tiles = ceil_div(N, kTile4Rows), k_tiles = ceil_div(K, kTile4K);
    const uint32_t local = blockIdx.x - g.wg_base;
    const uint32_t tile = local % n_tiles, row_tile = local / n_tiles;
    const uint32_t li = lane & 15, lq = lane >> 4;
    const uint32_t in_group = row_tile * 16 + li;
    const bool there = in_group < g.n_rows;
    const uint64_t row = (uint64_t)g.row0 + in_group;
    const uint8_t* w = a.arena + g.off + (uint64_t)tile * k_tiles * kTile4Bytes;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t kt = wave; kt < k_tiles; kt += WK) {
        const u32x4 codes = *(const u32x4*)(w + (uint64_t)kt * kTile4Bytes + lane * 16);
        const uint32_t sb = w[(uint64_t)kt * kTile4Bytes + kTile4Codes + lane];
        Operand<X> x;
        load_operand(x, a, row, kt * kTile4K + lq * 32, K, there);
        u32x4 wv[4];
        weights_of(codes, sb, wv);
#pragma unroll
        for (int p = Operand<X>::kParts - 1; p >= 0; --p)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wv[j]), __builtin_bit_cast(bf16x8, x.v[p][j]), acc, 0, 0, 0);
    }
    __shared__ f32x4 part[WK][64];
    part[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 1; i < WK; ++i) acc += part[i][lane];
    // lane l: row l % 16, outputs 4 (l / 16) .. + 3 of the tile
    const uint32_t n0 = tile * kTile4Rows + 4 * lq;
    if (!there || n0 >= N) return;
    const float* bias = g.has_bias ? (const float*)(a.arena + g.off + matrix4_tiles_bytes(N, K)) : nullptr;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) acc[i] = activate4(acc[i] + (bias && n0 + i < N ? bias[n0 + i] : 0.0f), a.act);
    Y* y = (Y*)a.y + row * a.y_stride + n0;
    if (n0 + 4 <= N) store4(y, acc);
    else
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) if (n0 + i < N) y[i] = (Y)acc[i];
}

template <typename X, typename Y>
hipError_t go(const Linear4Args& a, Linear4Shape, uint32_t grid, hipStream_t s)
{
    hipLaunchKernelGGL((linear4_kernel<X, Y, 4>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

Linear4Shape linear4_shape(uint64_t, uint32_t, uint32_t, uint32_t) { return Linear4Shape{1, 1, 4}; }

hipError_t launch_linear4(const Linear4Args& a, Linear4Shape shape, uint32_t x_dtype, uint32_t y_dtype, uint32_t grid, hipStream_t s)
{
    if (y_dtype == MT_BF16) {
        if (x_dtype == MT_MX8) return go<RowsMx8, __bf16>(a, shape, grid, s);
        return x_dtype == MT_BF16 ? go<RowsBf16, __bf16>(a, shape, grid, s) : go<RowsF32, __bf16>(a, shape, grid, s);
    }
    if (x_dtype == MT_MX8) return go<RowsMx8, float>(a, shape, grid, s);
    return x_dtype == MT_BF16 ? go<RowsBf16, float>(a, shape, grid, s) : go<RowsF32, float>(a, shape, grid, s);
}

}  // namespace mt
