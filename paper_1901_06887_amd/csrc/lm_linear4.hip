// mt_linear4: rows of many tenants times their 4-bit matrices.
//
// y[i][n] = act(b[n] + sum_k W[n][k] x[i][k]).  The weights are the row operand of the 16x16x32 bf16 matrix instruction, 16 rows of x the
// column operand: every e2m1 value times its scale is a bf16 value, every bf16 row value is itself one, an 8-bit one with its scale too, and an fp32
// one is the sum of three; so the products are exact and the sums fp32.  (The instruction that multiplies 4-bit and 8-bit values with their scales itself
// needs no conversions, but it keeps some 13 to 15 bits below the largest of the 128 products that it adds: blocks of small values vanish beside one of large ones.)
//
// Lane l of an operand holds output (or row) l % 16 and the 32 values of k block l / 16, which is how the weights lie in memory: one 16-byte load a lane
// is an operand, with one scale.  Rows are read in place, in the same order; those that do not exist are taken from the last one that does, and their
// columns of the product are never stored.
#include "lm_device.h"

namespace mt {
namespace {

enum Kind { kRowsF32, kRowsBf16, kRowsMx8 };
constexpr uint32_t row_size(Kind k) { return k == kRowsF32 ? 4 : k == kRowsBf16 ? 2 : 1; }

// fp32 as three bf16 values whose sum it is: the upper halves of what is left (bf16's smallest is 2^-133: bits below are lost).  An infinity or NaN is the first alone.
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

// Four of them, packed.
__device__ __forceinline__ void split3(const u32x4& x, uint32_t (&part)[3][2])
{
    const f32x4 f = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t lo[3], hi[3];
        split3(f[2 * i], lo); split3(f[2 * i + 1], hi);
#pragma unroll
        for (int q = 0; q < 3; ++q) part[q][i] = lo[q] >> 16 | hi[q];
    }
}

// The same at half the instructions where the wave has neither an infinity nor a NaN.  (Where the waves wait for this, through LDS: four tenants of 64 rows through
// 4096 x 4096 40.1 -> 35.1 us.  Where they wait for loads the branch costs more: one row 12.0 -> 12.5.)
__device__ __forceinline__ void split3_mostly_finite(const u32x4& x, uint32_t (&part)[3][2])
{
    const f32x4 f = __builtin_bit_cast(f32x4, x);
    const float zero = fmaf(f[3], 0.0f, fmaf(f[2], 0.0f, fmaf(f[1], 0.0f, f[0] * 0.0f)));
    if (__ballot(zero != 0.0f)) { split3(x, part); return; }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t p[3][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            p[0][h] = x[2 * i + h];               // (not a cast of the element of f: the compiler takes element 0 for every one)
            const float r = f[2 * i + h] - __builtin_bit_cast(float, p[0][h] & 0xffff0000u);
            p[1][h] = __builtin_bit_cast(uint32_t, r);
            p[2][h] = __builtin_bit_cast(uint32_t, r - __builtin_bit_cast(float, p[1][h] & 0xffff0000u));
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) part[q][i] = __builtin_amdgcn_perm(p[q][1], p[q][0], 0x07060302);       // the upper halves
    }
}

// 2^(byte - 127); the smallest is subnormal, the largest byte is NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte == 0xff ? 0x7fc00000u : byte ? byte << 23 : 0x00400000u); }
// Eight 8-bit values, scaled, as bf16.
__device__ __forceinline__ u32x4 eight_of(uint32_t lo, uint32_t hi, float s)
{
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true))};
}

// 16 bytes of a row, from any element's address.
template <Kind KIND> __device__ __forceinline__ u32x4 load16(const uint8_t* p)
{
    if constexpr (KIND == kRowsF32) return *(const Any<float>::vec16*)p;
    else if constexpr (KIND == kRowsBf16) return *(const Any<__bf16>::vec16*)p;
    else return *(const Any<uint8_t>::vec16*)p;
}

// The same from value `first` of a last k tile that is not whole: `left` values from `tile` on, zeros behind them.  A row of at least 16 bytes is read up to
// its end and shifted down: one load for every lane, where loads of single values would each wait for the one before.
template <Kind KIND> __device__ __forceinline__ u32x4 load16_last(const uint8_t* tile, uint32_t first, uint32_t left, uint32_t K)
{
    constexpr uint32_t es = row_size(KIND), kEach = 16 / es;
    u32x4 v;
    if (K >= kEach) {
        const int32_t over = max((int32_t)(first + kEach) - (int32_t)left, 0);      // values past the end (signed: from an unsigned difference the compiler took it that there are some)
        v = load16<KIND>(tile + (int64_t)((int32_t)first - over) * es);
        const uint32_t bytes = (uint32_t)min(over, (int32_t)kEach) * es;
        if (bytes & 8) v = u32x4{v[2], v[3], 0, 0};
        if (bytes & 4) v = u32x4{v[1], v[2], v[3], 0};
        if constexpr (es < 4)
            v = u32x4{__builtin_amdgcn_alignbyte(v[1], v[0], bytes & 3), __builtin_amdgcn_alignbyte(v[2], v[1], bytes & 3), __builtin_amdgcn_alignbyte(v[3], v[2], bytes & 3),
                      __builtin_amdgcn_alignbyte(0, v[3], bytes & 3)};
        if (bytes == 16) v = u32x4{0, 0, 0, 0};
    } else {
        v = u32x4{0, 0, 0, 0};
#pragma unroll
        for (uint32_t e = 0; e < kEach; ++e) {
            const uint32_t at = min(first + e, left - 1);
            uint32_t one;
            if constexpr (es == 4) one = ((const uint32_t*)tile)[at];
            else if constexpr (es == 2) one = ((const uint16_t*)tile)[at];
            else one = tile[at];
            if (first + e < left) v[e * es / 4] |= one << (8 * (e * es % 4));
        }
    }
    return v;
}

// A lane's 32 values of a row as they come from memory.
template <Kind KIND> struct RawRow {
    static constexpr uint32_t kVecs = row_size(KIND) * 2;      // of 16 bytes
    u32x4 v[kVecs];
    uint32_t scale;

    // tile: the row's values of the k tile; its scales likewise
    __device__ __forceinline__ void load(const uint8_t* tile, const uint8_t* scales, uint32_t lq)
    {
#pragma unroll
        for (uint32_t i = 0; i < kVecs; ++i) v[i] = load16<KIND>(tile + lq * (32 * row_size(KIND)) + 16 * i);
        if constexpr (KIND == kRowsMx8) scale = scales[lq];
    }
    __device__ __forceinline__ void load_last(const uint8_t* tile, const uint8_t* scales, uint32_t lq, uint32_t left, uint32_t K)
    {
#pragma unroll
        for (uint32_t i = 0; i < kVecs; ++i) v[i] = load16_last<KIND>(tile, lq * 32 + 16 / row_size(KIND) * i, left, K);
        if constexpr (KIND == kRowsMx8) scale = scales[min(lq, (left - 1) / MT_MX_BLOCK)];
    }
};

// ... the j-th eight of them as an operand of a 16x16x32 instruction (of three for fp32).
template <Kind KIND> struct RowOperand {
    static constexpr int kParts = KIND == kRowsF32 ? 3 : 1;
    u32x4 v[kParts];
    __device__ __forceinline__ RowOperand(const RawRow<KIND>& r, int j)
    {
        if constexpr (KIND == kRowsBf16) v[0] = r.v[j];
        else if constexpr (KIND == kRowsMx8) v[0] = eight_of(r.v[j / 2][2 * (j % 2)], r.v[j / 2][2 * (j % 2) + 1], scale_of(r.scale));
        else
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t part[3][2];
                split3(r.v[2 * j + h], part);
#pragma unroll
                for (int q = 0; q < 3; ++q) { v[q][2 * h] = part[q][0]; v[q][2 * h + 1] = part[q][1]; }
            }
    }
};

// A lane's 32 weights and their scale.
struct RawWeights { u32x4 codes; uint32_t scale; };
__device__ __forceinline__ RawWeights load_weights(const uint8_t* tile, uint32_t lane)
{
    return RawWeights{*(const u32x4*)(tile + lane * 16), tile[kTile4Codes + lane]};
}
// ... the j-th eight of them, scaled, as an operand.
__device__ __forceinline__ u32x4 weights_of(const RawWeights& r, int j)
{
    const float s = __builtin_bit_cast(float, r.scale << 23);
    const uint32_t c = r.codes[j];
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3))};
}

__device__ __forceinline__ f32x4 mfma(const u32x4& w, const u32x4& x, const f32x4& acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
}

// One k tile: NT tiles of 16 outputs times 16 rows.
template <Kind KIND, int NT> struct Step {
    RawWeights w[NT];
    RawRow<KIND> x;

    __device__ __forceinline__ void multiply(f32x4 (&acc)[NT]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const RowOperand<KIND> o(x, j);
            u32x4 wv[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) wv[n] = weights_of(w[n], j);
#pragma unroll
            for (int p = RowOperand<KIND>::kParts - 1; p >= 0; --p)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[n] = mfma(wv[n], o.v[p], acc[n]);
        }
    }
};

// NaN stays NaN in all.
__device__ __forceinline__ float relu4(float z) { return z < 0.0f ? 0.0f : z; }
__device__ __forceinline__ float gelu4(float z) { return 0.5f * z * erfcf(-0.70710678f * z); }
// For bf16, some 2^-17 of itself off at a third of the instructions: max(z, 0) - a q with a = |z| and q = normal tail beyond a = t P(t) exp(-a^2 / 2), t = 1 / (1 + 0.309 a); P is
// fitted to q exp(a^2 / 2) for the least largest relative error up to a = 14.6, beyond which a q is below bf16's smallest value.  2^24 moves from P to the exponential, which would
// else be 0 from a = 13.2 on.  Infinity minus 64 times 0 is infinity; -infinity times 0 is NaN, as in the other form.
__device__ __forceinline__ float gelu4_bf16(float z)
{
    constexpr float k = 0x1p-24f;
    const float a = fabsf(fminf(z, 64.0f));
    const float t = __builtin_amdgcn_rcpf(fmaf(0.309f, a, 1.0f));
    const float poly = t * (0.1234917f * k + t * (0.11965843f * k + t * (0.13500475f * k + t * (0.01144331f * k + t * (0.18512379f * k + t * (-0.07472409f * k))))));
    const float e = __builtin_amdgcn_exp2f(fmaf(-0.72134752f * a, a, 24.0f));             // (log2(e) / 2)
    return fmaf(-a, poly * e, relu4(z));
}

__device__ __forceinline__ void store4(__bf16* p, const f32x4& v) { *(Any<__bf16>::vec8*)p = Any<__bf16>::vec8{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }
__device__ __forceinline__ void store4(float* p, const f32x4& v) { *(Any<float>::vec16*)p = __builtin_bit_cast(u32x4, v); }

template <typename Y>
__device__ __forceinline__ void store_outputs(const Linear4Call& a, uint64_t row, uint32_t n0, uint32_t N, const f32x4& v)
{
    Y* y = (Y*)a.y + row * a.y_stride + n0;
    if (n0 + 4 <= N) store4(y, v);
    else
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) if (n0 + i < N) y[i] = (Y)v[i];
}

// The biases of four outputs, in loads that no branch holds up; past the last output, its own.
__device__ __forceinline__ f32x4 bias_of(const Linear4Call& a, const Group4& g, uint32_t n0)
{
    const float* p = (const float*)(a.arena + g.off + matrix4_tiles_bytes(g.N, g.K));
    f32x4 b;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) b[i] = p[min(n0 + i, g.N - 1)];
    return b;
}

// Four outputs of a row of the group: activation and store.
__device__ __forceinline__ void finish_tile(const Linear4Call& a, const Group4& g, uint32_t n0, uint32_t in_group, f32x4 v)
{
    if (in_group >= g.n_rows || n0 >= g.N) return;
    if (a.act == MT_ACT_GELU) {
        if (a.y_bf16) v = f32x4{gelu4_bf16(v[0]), gelu4_bf16(v[1]), gelu4_bf16(v[2]), gelu4_bf16(v[3])};
        else v = f32x4{gelu4(v[0]), gelu4(v[1]), gelu4(v[2]), gelu4(v[3])};
    } else if (a.act == MT_ACT_RELU) v = f32x4{relu4(v[0]), relu4(v[1]), relu4(v[2]), relu4(v[3])};
    if (a.y_bf16) store_outputs<__bf16>(a, (uint64_t)g.row0 + in_group, n0, g.N, v);
    else store_outputs<float>(a, (uint64_t)g.row0 + in_group, n0, g.N, v);
}

// A workgroup's group: the last one that starts at or before it.  (What a kernel reads of its arguments is asked for in one go and waited for here: loads
// where they are used are as many trips to memory one after the other, some 500 clocks each in a launch's first workgroups.)
template <uint32_t GROUPS>
__device__ __forceinline__ Group4 group_of(const Linear4Args<GROUPS>& args, uint32_t lane)
{
    const Linear4Call& a = args.call;
    Group4 g = args.groups[0];
    asm volatile("" :: "s"(a.arena), "s"(a.x), "s"(a.x_scales), "s"(a.y), "s"(a.x_stride), "s"(a.x_scales_stride), "s"(a.y_stride), "s"(a.act), "s"(a.n_groups), "s"(a.y_bf16),
                 "s"(g.off), "s"(g.N), "s"(g.K), "s"(g.row0), "s"(g.n_rows));
    if (a.n_groups > 1) {
        const bool starts = lane < a.n_groups && args.groups[lane < a.n_groups ? lane : 0].wg_base <= blockIdx.x;
        g = args.groups[__builtin_amdgcn_readfirstlane(__popcll(__ballot(starts)) - 1)];
        asm volatile("" :: "s"(g.off), "s"(g.N), "s"(g.K), "s"(g.row0), "s"(g.n_rows), "s"(g.wg_base));
    }
    return g;
}

constexpr int kWaves4 = 4;      // waves of a workgroup: they share the k tiles and add their sums up through LDS

// A workgroup serves 16 NT outputs of 16 rows of a group; a wave asks for DEPTH k tiles at a time, the next ones before it multiplies.  The weights' bytes bound it,
// for small matrices the launch and two trips to memory: one bf16 row through 4096 x 65536 26.2 us (5.5 TB/s), through 1024 x 1024 3.4 us; 64 tenants of one to
// four 8-bit rows through 1024 x 1024 9.1 us (4.0 TB/s).  Waves matter more than depth: with registers for two waves a SIMD instead of three and four the last took 10.2,
// 40 tenants of 64 fp32 rows through 448 x 960 50 instead of 28; 8 or 16 waves to a workgroup, or deeper walks, gave nothing.
template <Kind KIND, int NT, int DEPTH, uint32_t GROUPS>
__global__ void __launch_bounds__(kWaves4 * 64, KIND == kRowsF32 ? 3 : 2) linear4_kernel(Linear4Args<GROUPS> args)
{
    const Linear4Call& a = args.call;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Group4 g = group_of(args, lane);
    const uint32_t N = g.N, K = g.K;
    const uint32_t n_tiles = ceil_div(N, kTile4Rows), k_tiles = ceil_div(K, kTile4K), n_slabs = ceil_div(n_tiles, NT);
    const uint32_t local = blockIdx.x - g.wg_base;
    const uint32_t slab = local % n_slabs, first_row = local / n_slabs * kTile4Rows;
    const uint32_t li = lane & 15, lq = lane >> 4;
    const uint8_t* w[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) w[n] = a.arena + g.off + (uint64_t)min(slab * NT + n, n_tiles - 1) * k_tiles * kTile4Bytes;
    const uint64_t row = (uint64_t)g.row0 + min(first_row + li, g.n_rows - 1);
    const uint8_t* x = (const uint8_t*)a.x + row * a.x_stride * row_size(KIND);
    const uint8_t* xs = a.x_scales + row * a.x_scales_stride;
    f32x4 acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const f32x4 bias = bias_of(a, g, (slab * NT + wave) * kTile4Rows + 4 * lq);       // for the tile that this wave finishes

    // whole k tiles: this wave's are wave, wave + 4, ...
    const uint32_t whole = K / kTile4K;
    Step<KIND, NT> at[2][DEPTH];
    const auto ask = [&](Step<KIND, NT> (&to)[DEPTH], uint32_t kt) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const uint32_t t = min(kt + d * kWaves4, whole - 1);
#pragma unroll
            for (int n = 0; n < NT; ++n) to[d].w[n] = load_weights(w[n] + (uint64_t)t * kTile4Bytes, lane);
            to[d].x.load(x + t * (kTile4K * row_size(KIND)), xs + t * 4, lq);
        }
    };
    const auto use = [&](const Step<KIND, NT> (&of)[DEPTH], uint32_t kt) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) if (d == 0 || kt + d * kWaves4 < whole) of[d].multiply(acc);
    };
    constexpr uint32_t kStride = DEPTH * kWaves4;
    if (wave < whole) {
        uint32_t kt = wave;
        ask(at[0], kt);
        while (true) {
            if (kt + kStride < whole) ask(at[1], kt + kStride);
            use(at[0], kt);
            kt += kStride;
            if (kt >= whole) break;
            if (kt + kStride < whole) ask(at[0], kt + kStride);
            use(at[1], kt);
            kt += kStride;
            if (kt >= whole) break;
        }
    }
    if (whole < k_tiles && whole % kWaves4 == wave) {           // the last one, where it is not whole
        Step<KIND, NT> last;
#pragma unroll
        for (int n = 0; n < NT; ++n) last.w[n] = load_weights(w[n] + (uint64_t)whole * kTile4Bytes, lane);
        last.x.load_last(x + (uint64_t)whole * (kTile4K * row_size(KIND)), xs + whole * 4, lq, K - whole * kTile4K, K);
        last.multiply(acc);
    }

    // tile n is finished by wave n
    static_assert(NT <= kWaves4, "a wave finishes one tile at most");
    __shared__ f32x4 part[kWaves4][NT][64];
#pragma unroll
    for (int n = 0; n < NT; ++n) if (n != (int)wave) part[wave][n][lane] = acc[n];
    lds_barrier();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n != (int)wave) continue;
        f32x4 v = acc[n] + bias;
#pragma unroll
        for (int o = 1; o < kWaves4; ++o) v += part[(wave + o) % kWaves4][n][lane];
        // lane l: row l % 16, outputs 4 (l / 16) .. + 3 of the tile
        finish_tile(a, g, (slab * NT + n) * kTile4Rows + 4 * lq, first_row + li, v);
    }
}

// ---- many rows: rows through LDS ----------------------------------------------------------------
// 16 RT rows and 128 outputs to a workgroup of eight waves: 64 outputs (slab) x a quarter of the k tiles to each.  The two waves of a quarter fetch its rows
// together, 16 bytes a lane along the rows (read in place by operands, a load would touch 64 lines; 512 rows through 4096 x 4096 took 44.6 us that way), and
// put them into LDS as bf16 operands: chunk c (eight values) of row i at slot i ^ c of its sixteen, so that neither the stores along a row nor the loads
// down the rows meet in a bank.  Two buffers, so one barrier for a k tile.  The weights go from memory to registers two k tiles ahead.
// 512 bf16 rows through 4096 x 4096 21.5 us (0.80 PFLOP/s), eight tenants of 37 to 64 8-bit rows through 4096 x 4096 with GELU 24.6 us.  Of the latter's 50 thousand clocks
// 7 pass before the first product (arguments, then rows and weights), 33 in eight rounds of four k tiles, half of them MFMAs (the rest: conversion of the weights, which
// every wave does for its 64 outputs, LDS stores, the barrier), 10 at the join and the activation.
constexpr int kSlabs = 2, kQuarters = 4, kNt = 4;

template <Kind KIND, int RT> struct RowFetch {
    static constexpr uint32_t kPer = 16 / row_size(KIND), kAcross = kTile4K / kPer;         // values of a load; loads along a row
    static constexpr uint32_t kRowsAtOnce = 128 / kAcross, kPasses = 16 * RT / kRowsAtOnce;
    const uint8_t* p[kPasses];
    const uint8_t* ps[KIND == kRowsMx8 ? kPasses : 1];
    u32x4 v[kPasses];
    uint32_t scale[KIND == kRowsMx8 ? kPasses : 1];
    uint32_t u, row0;              // which load along the row, and row, this thread starts with

    __device__ __forceinline__ RowFetch(const Linear4Call& a, const Group4& g, uint32_t first_row, uint32_t t) : u(t % kAcross), row0(t / kAcross)
    {
#pragma unroll
        for (uint32_t i = 0; i < kPasses; ++i) {
            const uint64_t row = (uint64_t)g.row0 + min(first_row + row0 + i * kRowsAtOnce, g.n_rows - 1);
            p[i] = (const uint8_t*)a.x + row * a.x_stride * row_size(KIND);
            if constexpr (KIND == kRowsMx8) ps[i] = a.x_scales + row * a.x_scales_stride;
        }
    }
    __device__ __forceinline__ void ask(uint32_t kt)
    {
#pragma unroll
        for (uint32_t i = 0; i < kPasses; ++i) {
            v[i] = load16<KIND>(p[i] + kt * (kTile4K * row_size(KIND)) + u * 16);
            if constexpr (KIND == kRowsMx8) scale[i] = ps[i][kt * (kTile4K / MT_MX_BLOCK) + u / 2];
        }
    }
    __device__ __forceinline__ void ask_last(uint32_t kt, uint32_t left, uint32_t K)
    {
#pragma unroll
        for (uint32_t i = 0; i < kPasses; ++i) {
            v[i] = load16_last<KIND>(p[i] + kt * (kTile4K * row_size(KIND)), u * kPer, left, K);
            if constexpr (KIND == kRowsMx8) scale[i] = ps[i][kt * (kTile4K / MT_MX_BLOCK) + min(u / 2, (left - 1) / MT_MX_BLOCK)];
        }
    }
    static __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t c)      // in 16 bytes
    {
        return ((row / 16 * 4 + c % 4) * 4 + c / 4) * 16 + (row % 16 ^ c);
    }
    __device__ __forceinline__ void put(u32x4* to) const
    {
#pragma unroll
        for (uint32_t i = 0; i < kPasses; ++i) {
            const uint32_t row = row0 + i * kRowsAtOnce;
            if constexpr (KIND == kRowsBf16) to[place(row, u)] = v[i];
            else if constexpr (KIND == kRowsF32) {
                uint32_t part[3][2];
                split3_mostly_finite(v[i], part);
#pragma unroll
                for (uint32_t q = 0; q < 3; ++q) *((u32x2*)(to + q * (16 * RT * 16) + place(row, u / 2)) + u % 2) = u32x2{part[q][0], part[q][1]};
            } else {
                const float s = scale_of(scale[i]);
                to[place(row, 2 * u)] = eight_of(v[i][0], v[i][1], s);
                to[place(row, 2 * u + 1)] = eight_of(v[i][2], v[i][3], s);
            }
        }
    }
};

template <Kind KIND, int RT>
__global__ void __launch_bounds__(512) linear4_rows_kernel(Linear4Args<kGroups4> args)
{
    const Linear4Call& a = args.call;
    extern __shared__ __attribute__((aligned(16))) u32x4 lds[];
    constexpr uint32_t kParts = KIND == kRowsF32 ? 3 : 1, kPartVecs = 16 * RT * 16, kTileVecs = kParts * kPartVecs;      // a k tile of the rows, in 16 bytes
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t quarter = wave / kSlabs, li = lane & 15, lq = lane >> 4;
    const Group4 g = group_of(args, lane);
    const uint32_t N = g.N, K = g.K;
    const uint32_t n_tiles = ceil_div(N, kTile4Rows), k_tiles = ceil_div(K, kTile4K), n_wide = ceil_div(n_tiles, kNt * kSlabs), chunks = ceil_div(g.n_rows, 16 * RT);
    // workgroups eight apart share an XCD: they take the same outputs of one chunk of rows after the other
    uint32_t wide = blockIdx.x - g.wg_base, chunk = 0;
    if (chunks > 1) {
        const uint32_t local = wide, in_eights = n_wide / 8 * 8 * chunks;
        if (local < in_eights) { const uint32_t eighth = local / 8, n = eighth / chunks; wide = n * 8 + local % 8; chunk = eighth - n * chunks; }
        else { const uint32_t rest = local - in_eights, n = n_wide % 8; chunk = rest / n; wide = n_wide - n + (rest - chunk * n); }
    }
    const uint32_t slab = wide * kSlabs + wave % kSlabs, first_row = chunk * (16 * RT);
    const uint8_t* w[kNt];
#pragma unroll
    for (int n = 0; n < kNt; ++n) w[n] = a.arena + g.off + (uint64_t)min(slab * kNt + n, n_tiles - 1) * k_tiles * kTile4Bytes;
    RowFetch<KIND, RT> x(a, g, first_row, threadIdx.x % (64 * kSlabs));
    f32x4 acc[kNt][RT];
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[n][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const auto ask_weights = [&](RawWeights (&to)[kNt], uint32_t kt) {
#pragma unroll
        for (int n = 0; n < kNt; ++n) to[n] = load_weights(w[n] + (uint64_t)kt * kTile4Bytes, lane);
    };
    const auto multiply = [&](const RawWeights (&wt)[kNt], const u32x4* tile) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 wv[kNt];
#pragma unroll
            for (int n = 0; n < kNt; ++n) wv[n] = weights_of(wt[n], j);
#pragma unroll
            for (int p = kParts - 1; p >= 0; --p) {
                u32x4 o[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) o[r] = tile[p * kPartVecs + ((r * 4 + j) * 4 + lq) * 16 + (li ^ (lq * 4 + j))];
#pragma unroll
                for (int n = 0; n < kNt; ++n)
#pragma unroll
                    for (int r = 0; r < RT; ++r) acc[n][r] = mfma(wv[n], o[r], acc[n][r]);
            }
        }
    };
    f32x4 bias[kNt * RT / kQuarters];
#pragma unroll
    for (int i = 0; i < kNt * RT / kQuarters; ++i) bias[i] = bias_of(a, g, (slab * kNt + (i * kQuarters + quarter) / RT) * kTile4Rows + 4 * lq);
    // Whole k tiles, in rounds of four.  A quarter whose turn finds none left asks for the last one again and multiplies nothing: with loads inside
    // of conditions the compiler's counts of what is in flight would make every round wait for all of it.
    u32x4* tiles = lds + quarter * 2 * kTileVecs;
    const uint32_t whole = K / kTile4K, rounds = ceil_div(whole, kQuarters);
    if (rounds) {
        RawWeights ws[2][kNt];
        const auto nth = [&](uint32_t round) { return min(quarter + round * kQuarters, whole - 1); };
        const auto step = [&](RawWeights (&wt)[kNt], uint32_t round) {
            u32x4* tile = tiles + round % 2 * kTileVecs;
            x.put(tile);
            x.ask(nth(round + 1));
            lds_barrier();
            if (quarter + round * kQuarters < whole) multiply(wt, tile);
            ask_weights(wt, nth(round + 2));
        };
        ask_weights(ws[0], nth(0));
        x.ask(nth(0));
        ask_weights(ws[1], nth(1));
        for (uint32_t round = 0;;) {
            step(ws[0], round);
            if (++round == rounds) break;
            step(ws[1], round);
            if (++round == rounds) break;
        }
    }
    if (whole < k_tiles) {
        RawWeights wl[kNt];
        ask_weights(wl, whole);
        const bool mine = whole % kQuarters == quarter;
        if (mine) x.ask_last(whole, K - whole * kTile4K, K);
        lds_barrier();
        if (mine) x.put(tiles);
        lds_barrier();
        if (mine) multiply(wl, tiles);
    }
    // quarter q finishes the tiles t with t % 4 = q of its slab, with the sums of the other quarters
    lds_barrier();
    f32x4* part = (f32x4*)lds;
    const auto at = [&](uint32_t q, uint32_t t) { return ((q * kSlabs + wave % kSlabs) * (kNt * RT) + t) * 64 + lane; };
#pragma unroll
    for (int t = 0; t < kNt * RT; ++t) if (t % kQuarters != (int)quarter) part[at(quarter, t)] = acc[t / RT][t % RT];
    lds_barrier();
#pragma unroll
    for (int t = 0; t < kNt * RT; ++t) {
        if (t % kQuarters != (int)quarter) continue;
        f32x4 v = acc[t / RT][t % RT] + bias[t / kQuarters];
#pragma unroll
        for (int o = 1; o < kQuarters; ++o) v += part[at((quarter + o) % kQuarters, t)];
        finish_tile(a, g, (slab * kNt + t / RT) * kTile4Rows + 4 * lq, first_row + 16 * (t % RT) + li, v);
    }
}
// both buffers of rows, or the sums at the end
template <Kind KIND, int RT> constexpr uint32_t rows_lds()
{
    constexpr uint32_t rows = kQuarters * 2 * 16 * RT * 256 * (KIND == kRowsF32 ? 3 : 1), sums = kQuarters * kSlabs * (kNt * RT) * 1024;
    static_assert(rows <= 160 * 1024 && sums <= 160 * 1024, "LDS");
    return rows > sums ? rows : sums;
}

template <Kind KIND, int NT, int DEPTH>
hipError_t go(const Linear4Args<kGroups4>& a, uint32_t grid, hipStream_t s)
{
    if (a.call.n_groups <= kFewGroups4) return launch(linear4_kernel<KIND, NT, DEPTH, kFewGroups4>, dim3(grid), kWaves4 * 64, 0, s, a);
    return launch(linear4_kernel<KIND, NT, DEPTH, kGroups4>, dim3(grid), kWaves4 * 64, 0, s, a);
}

template <Kind KIND, int RT>
hipError_t go_rows(const Linear4Args<kGroups4>& a, uint32_t grid, hipStream_t s)
{
    return launch(linear4_rows_kernel<KIND, RT>, dim3(grid), 512, rows_lds<KIND, RT>(), s, a);
}

template <Kind KIND>
hipError_t choose(const Linear4Args<kGroups4>& a, Linear4Shape shape, uint32_t grid, hipStream_t s)
{
    if (!shape.through_lds) return shape.nt == 1 ? go<KIND, 1, KIND == kRowsF32 ? 1 : 4>(a, grid, s) : go<KIND, 4, 1>(a, grid, s);
    if constexpr (KIND == kRowsF32) return go_rows<KIND, 1>(a, grid, s);
    else return shape.rt == 2 ? go_rows<KIND, 2>(a, grid, s) : go_rows<KIND, 4>(a, grid, s);
}

template <Kind KIND, int RT>
hipError_t prepare_rows() { return hipFuncSetAttribute((const void*)linear4_rows_kernel<KIND, RT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)rows_lds<KIND, RT>()); }

}  // namespace

// Kernel times (us) of the three forms, 16 x 16 tiles with a workgroup for 16 outputs / for 64 / rows through LDS:
//   bf16, 24 rows through 4864 x 832 8.4 / 8.7 / 13.0, three tenants of them 14.3 / 9.7 / 13.7; 16 rows through 4096 x 4096 7.2 / 8.2 / 11.9, 24 rows 9.8 / 8.3 / 11.9,
//   64 18.6 / 8.7 / 18.5, two tenants of those 34.9 / 14.2 / 18.8, four 66.9 / 24.6 / 20.6; 40 tenants of 64 rows through 448 x 960 84 / 17.0 / 20.2; one row through
//   4096 x 8192 6.2 / 6.7, x 32768 16.7 / 12.8
//   fp32, 64 rows through 4096 x 4096 40.9 / 18.2 / 18.6, two tenants 76.3 / 30.3 / 18.4; 8 tenants of 64 rows through 1024 x 1024 24.3 / 11.8 / 9.0; one row
//   through 4096 x 4096 12.0 / 14.3, x 8192 19.1 / 14.8, x 32768 63.2 / 26.5 / 18.4
// So rows go through LDS where that makes half as many workgroups as there are compute units (fp32, whose every value is split: three quarters, and for few
// rows too) of two k tiles or more to a wave; else a workgroup takes 64 outputs where workgroups for 16 would be more than the compute units, or four times as many
// where few rows are read and not split.
Linear4Shape linear4_shape(uint64_t row_tiles, uint32_t most_rows, uint32_t most_k, uint32_t n_cus, uint32_t x_dtype)
{
    const bool f32 = x_dtype == MT_F32;
    Linear4Shape s;
    s.rt = most_rows <= 16 || f32 ? 1 : most_rows <= 32 ? 2 : 4;
    s.nt = kNt * kSlabs;
    s.through_lds = (f32 || most_rows > 16) && row_tiles / (s.nt * s.rt) >= (f32 ? 3 * n_cus / 4 : n_cus / 2) && most_k >= 2 * kQuarters * kTile4K;
    if (!s.through_lds) {
        s.rt = 1;
        s.nt = row_tiles > (most_rows > 4 || f32 ? n_cus : 4 * n_cus - 1) ? 4 : 1;
    }
    return s;
}

hipError_t prepare_linear4()
{
    hipError_t e = prepare_rows<kRowsF32, 1>();
    if (e == hipSuccess) e = prepare_rows<kRowsBf16, 2>();
    if (e == hipSuccess) e = prepare_rows<kRowsBf16, 4>();
    if (e == hipSuccess) e = prepare_rows<kRowsMx8, 2>();
    return e == hipSuccess ? prepare_rows<kRowsMx8, 4>() : e;
}

hipError_t launch_linear4(const Linear4Args<kGroups4>& a, Linear4Shape shape, uint32_t x_dtype, uint32_t grid, hipStream_t s)
{
    if (x_dtype == MT_MX8) return choose<kRowsMx8>(a, shape, grid, s);
    return x_dtype == MT_BF16 ? choose<kRowsBf16>(a, shape, grid, s) : choose<kRowsF32>(a, shape, grid, s);
}

}  // namespace mt
