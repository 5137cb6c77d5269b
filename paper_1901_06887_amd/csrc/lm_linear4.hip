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

// 2^(byte - 127); the smallest is subnormal, the largest byte is NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte == 0xff ? 0x7fc00000u : byte ? byte << 23 : 0x00400000u); }
// Eight 8-bit values, scaled, as bf16.
__device__ __forceinline__ u32x4 eight_of(uint32_t lo, uint32_t hi, float s)
{
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true))};
}

// A lane's 32 values of a row as they come from memory.
template <Kind KIND> struct RawRow {
    static constexpr uint32_t kVecs = row_size(KIND) * 2;      // of 16 bytes
    u32x4 v[kVecs];
    uint32_t scale;

    // p: the lane's k block
    __device__ __forceinline__ void load(const uint8_t* p, const uint8_t* scale_at)
    {
#pragma unroll
        for (uint32_t i = 0; i < kVecs; ++i) {
            const uint8_t* q = p + 16 * i;
            if constexpr (KIND == kRowsF32) v[i] = *(const Any<float>::vec16*)q;
            else if constexpr (KIND == kRowsBf16) v[i] = *(const Any<__bf16>::vec16*)q;
            else v[i] = *(const Any<uint8_t>::vec16*)q;
        }
        if constexpr (KIND == kRowsMx8) scale = *scale_at;
    }

    // The last k tile, of `left` values from k block 0 on: zeros behind them.
    __device__ __forceinline__ void load_last(const uint8_t* p, const uint8_t* scale_at, uint32_t lq, uint32_t left)
    {
        constexpr uint32_t es = row_size(KIND), kEach = 16 / es;                // values of a vector
#pragma unroll
        for (uint32_t i = 0; i < kVecs; ++i) {
            const uint32_t first = lq * 32 + kEach * i;     // ... its first one
            const uint8_t* q = p + 16 * i;
            v[i] = u32x4{0, 0, 0, 0};
            if (first + kEach <= left) {
                if constexpr (KIND == kRowsF32) v[i] = *(const Any<float>::vec16*)q;
                else if constexpr (KIND == kRowsBf16) v[i] = *(const Any<__bf16>::vec16*)q;
                else v[i] = *(const Any<uint8_t>::vec16*)q;
            } else if (first < left) {
#pragma unroll
                for (uint32_t e = 0; e < kEach; ++e)
                    if (first + e < left) {
                        if constexpr (es == 4) v[i][e] = ((const uint32_t*)q)[e];
                        else if constexpr (es == 2) v[i][e / 2] |= (uint32_t)((const uint16_t*)q)[e] << (16 * (e % 2));
                        else v[i][e / 4] |= (uint32_t)q[e] << (8 * (e % 4));
                    }
            }
        }
        if constexpr (KIND == kRowsMx8) scale = lq * 32 < left ? *scale_at : 127;
    }
};

// ... and as operands of four 16x16x32 instructions (times three for fp32).
template <Kind KIND> struct RowOperand {
    static constexpr int kParts = KIND == kRowsF32 ? 3 : 1;
    u32x4 v[kParts][4];
    __device__ __forceinline__ explicit RowOperand(const RawRow<KIND>& r)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (KIND == kRowsBf16) v[0][j] = r.v[j];
            else if constexpr (KIND == kRowsF32) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 f = __builtin_bit_cast(f32x4, r.v[2 * j + h]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t lo[3], hi[3];
                        split3(f[2 * i], lo); split3(f[2 * i + 1], hi);
#pragma unroll
                        for (int q = 0; q < 3; ++q) v[q][j][2 * h + i] = lo[q] >> 16 | hi[q];
                    }
                }
            } else if constexpr (KIND == kRowsMx8) {
                v[0][j] = eight_of(r.v[j / 2][2 * (j % 2)], r.v[j / 2][2 * (j % 2) + 1], scale_of(r.scale));
            }
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

// One k tile: NT tiles of 16 outputs, RT tiles of 16 rows.
template <Kind KIND, int RT, int NT> struct Step {
    RawWeights w[NT];
    RawRow<KIND> x[RT];

    __device__ __forceinline__ void multiply(f32x4 (&acc)[NT][RT]) const
    {
        u32x4 wv[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) wv[n][j] = weights_of(w[n], j);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const RowOperand<KIND> o(x[r]);
#pragma unroll
            for (int p = RowOperand<KIND>::kParts - 1; p >= 0; --p)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[n][r] = mfma(wv[n][j], o.v[p][j], acc[n][r]);
        }
    }
};

// NaN stays NaN in both.  GELU: the library's erfc where fp32 is written; for bf16 the formula of the fully-connected layers (some 1e-7 off, a quarter of
// the instructions), kept from multiplying an infinity by 0.
__device__ __forceinline__ float activate4(float z, uint32_t act, uint32_t to_bf16)
{
    if (act == MT_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (!to_bf16) return 0.5f * z * erfcf(-0.70710678f * z);
    return fabsf(z) < 64.0f ? gelu(z) : z > 0.0f ? z : z < 0.0f ? -0.0f : z;
}

__device__ __forceinline__ void store4(__bf16* p, const f32x4& v) { *(Any<__bf16>::vec8*)p = Any<__bf16>::vec8{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }
__device__ __forceinline__ void store4(float* p, const f32x4& v) { *(Any<float>::vec16*)p = __builtin_bit_cast(u32x4, v); }

template <typename Y>
__device__ __forceinline__ void store_outputs(const Linear4Args& a, uint64_t row, uint32_t n0, uint32_t N, const f32x4& v)
{
    Y* y = (Y*)a.y + row * a.y_stride + n0;
    if (n0 + 4 <= N) store4(y, v);
    else
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) if (n0 + i < N) y[i] = (Y)v[i];
}

// The biases of four outputs; zeros where there are none.
__device__ __forceinline__ f32x4 bias_of(const Linear4Args& a, const Group4& g, uint32_t n0)
{
    f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!g.has_bias) return b;
    const float* p = (const float*)(a.arena + g.off + matrix4_tiles_bytes(g.N, g.K));
    if (n0 + 4 <= g.N) b = __builtin_bit_cast(f32x4, *(const Any<float>::vec16*)(p + n0));
    else
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) if (n0 + i < g.N) b[i] = p[n0 + i];
    return b;
}

// Four outputs of a row of the group: activation and store.
__device__ __forceinline__ void finish_tile(const Linear4Args& a, const Group4& g, uint32_t n0, uint32_t in_group, f32x4 v)
{
    if (in_group >= g.n_rows || n0 >= g.N) return;
    if (a.act != MT_ACT_NONE) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = activate4(v[i], a.act, a.y_bf16);
    }
    if (a.y_bf16) store_outputs<__bf16>(a, (uint64_t)g.row0 + in_group, n0, g.N, v);
    else store_outputs<float>(a, (uint64_t)g.row0 + in_group, n0, g.N, v);
}

// A workgroup's group: the last one that starts at or before it.
__device__ __forceinline__ uint32_t group_of(const Linear4Args& a, uint32_t lane)
{
    if (a.n_groups == 1) return 0;
    const bool starts = lane < a.n_groups && a.groups[lane < a.n_groups ? lane : 0].wg_base <= blockIdx.x;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(starts)) - 1);
}

constexpr int kWaves4 = 4;      // waves of a workgroup: they share the k tiles and add their sums up through LDS

// A workgroup serves 16 NT outputs of 16 RT rows of a group; a wave asks for DEPTH k tiles at a time, the next ones before it multiplies.
template <Kind KIND, int RT, int NT, int DEPTH>
__global__ void __launch_bounds__(kWaves4 * 64) linear4_kernel(Linear4Args a)
{
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Group4& g = a.groups[group_of(a, lane)];
    const uint32_t N = g.N, K = g.K;
    const uint32_t n_tiles = ceil_div(N, kTile4Rows), k_tiles = ceil_div(K, kTile4K), n_slabs = ceil_div(n_tiles, NT);
    const uint32_t local = blockIdx.x - g.wg_base;
    const uint32_t slab = local % n_slabs, first_row = local / n_slabs * (16 * RT);
    const uint32_t li = lane & 15, lq = lane >> 4;
    const uint8_t* w[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) w[n] = a.arena + g.off + (uint64_t)min(slab * NT + n, n_tiles - 1) * k_tiles * kTile4Bytes;
    const uint8_t *x[RT], *xs[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const uint64_t row = (uint64_t)g.row0 + min(first_row + 16 * r + li, g.n_rows - 1);
        x[r] = (const uint8_t*)a.x + row * a.x_stride * row_size(KIND) + lq * (32 * row_size(KIND));
        xs[r] = a.x_scales + row * a.x_scales_stride + lq;
    }
    f32x4 acc[NT][RT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[n][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // whole k tiles: this wave's are wave, wave + 4, ...
    const uint32_t whole = K / kTile4K;
    Step<KIND, RT, NT> at[2][DEPTH];
    const auto ask = [&](Step<KIND, RT, NT> (&to)[DEPTH], uint32_t kt) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const uint32_t t = min(kt + d * kWaves4, whole - 1);
#pragma unroll
            for (int n = 0; n < NT; ++n) to[d].w[n] = load_weights(w[n] + (uint64_t)t * kTile4Bytes, lane);
#pragma unroll
            for (int r = 0; r < RT; ++r) to[d].x[r].load(x[r] + t * (kTile4K * row_size(KIND)), xs[r] + t * 4);
        }
    };
    const auto use = [&](const Step<KIND, RT, NT> (&of)[DEPTH], uint32_t kt) {
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
        Step<KIND, RT, NT> last;
#pragma unroll
        for (int n = 0; n < NT; ++n) last.w[n] = load_weights(w[n] + (uint64_t)whole * kTile4Bytes, lane);
#pragma unroll
        for (int r = 0; r < RT; ++r) last.x[r].load_last(x[r] + (uint64_t)whole * (kTile4K * row_size(KIND)), xs[r] + whole * 4, lq, K - whole * kTile4K);
        last.multiply(acc);
    }

    // tile t of the NT x RT is finished by wave t % 4
    f32x4 bias[(NT * RT + kWaves4 - 1) / kWaves4];
#pragma unroll
    for (int i = 0; i < (NT * RT + kWaves4 - 1) / kWaves4; ++i) bias[i] = bias_of(a, g, (slab * NT + (i * kWaves4 + wave) / RT) * kTile4Rows + 4 * lq);
    __shared__ f32x4 part[kWaves4][NT * RT][64];
#pragma unroll
    for (int t = 0; t < NT * RT; ++t) if (t % kWaves4 != (int)wave) part[wave][t][lane] = acc[t / RT][t % RT];
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NT * RT; ++t) {
        if (t % kWaves4 != (int)wave) continue;
        f32x4 v = acc[t / RT][t % RT] + bias[t / kWaves4];
#pragma unroll
        for (int o = 1; o < kWaves4; ++o) v += part[(wave + o) % kWaves4][t][lane];
        finish_tile(a, g, (slab * NT + t / RT) * kTile4Rows + 4 * lq, first_row + 16 * (t % RT) + li, v);
    }
}

// ---- many rows: rows through LDS ----------------------------------------------------------------
// 16 RT rows and 128 outputs to a workgroup of eight waves: 64 outputs (slab) x a quarter of the k tiles to each.  The two waves of a quarter fetch its rows
// together, 16 bytes a lane along the rows (read in place by operands, a load would touch 64 lines; 512 rows through 4096 x 4096 took 44.6 us that way), and
// put them into LDS as bf16 operands: chunk c (eight values) of row i at slot i ^ c of its sixteen, so that neither the stores along a row nor the loads
// down the rows meet in a bank.  Two buffers, so one barrier for a k tile.  The weights go from memory to registers two k tiles ahead.
constexpr int kSlabs = 2, kQuarters = 4, kNt = 4;

template <Kind KIND, int RT> struct RowFetch {
    static constexpr uint32_t kPer = 16 / row_size(KIND), kAcross = kTile4K / kPer;         // values of a load; loads along a row
    static constexpr uint32_t kRowsAtOnce = 128 / kAcross, kPasses = 16 * RT / kRowsAtOnce;
    const uint8_t* p[kPasses];
    const uint8_t* ps[KIND == kRowsMx8 ? kPasses : 1];
    u32x4 v[kPasses];
    uint32_t scale[KIND == kRowsMx8 ? kPasses : 1];
    uint32_t u, row0;              // which load along the row, and row, this thread starts with

    __device__ __forceinline__ RowFetch(const Linear4Args& a, const Group4& g, uint32_t first_row, uint32_t t) : u(t % kAcross), row0(t / kAcross)
    {
#pragma unroll
        for (uint32_t i = 0; i < kPasses; ++i) {
            const uint64_t row = (uint64_t)g.row0 + min(first_row + row0 + i * kRowsAtOnce, g.n_rows - 1);
            p[i] = (const uint8_t*)a.x + row * a.x_stride * row_size(KIND) + u * 16;
            if constexpr (KIND == kRowsMx8) ps[i] = a.x_scales + row * a.x_scales_stride + u / 2;
        }
    }
    __device__ __forceinline__ void ask(uint32_t kt)
    {
#pragma unroll
        for (uint32_t i = 0; i < kPasses; ++i) {
            const uint8_t* q = p[i] + kt * (kTile4K * row_size(KIND));
            if constexpr (KIND == kRowsBf16) v[i] = *(const Any<__bf16>::vec16*)q;
            else { v[i] = *(const Any<uint8_t>::vec16*)q; scale[i] = ps[i][kt * (kTile4K / MT_MX_BLOCK)]; }
        }
    }
    // The last k tile where it is not whole, `left` values long: zeros behind them.
    __device__ __forceinline__ void ask_last(uint32_t kt, uint32_t left)
    {
#pragma unroll
        for (uint32_t i = 0; i < kPasses; ++i) {
            const uint8_t* q = p[i] + kt * (kTile4K * row_size(KIND));
            v[i] = u32x4{0, 0, 0, 0};
#pragma unroll
            for (uint32_t e = 0; e < kPer; ++e)
                if (u * kPer + e < left) {
                    if constexpr (KIND == kRowsBf16) v[i][e / 2] |= (uint32_t)((const uint16_t*)q)[e] << (16 * (e % 2));
                    else v[i][e / 4] |= (uint32_t)q[e] << (8 * (e % 4));
                }
            if constexpr (KIND == kRowsMx8) scale[i] = u * kPer < left ? ps[i][kt * (kTile4K / MT_MX_BLOCK)] : 127;
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
            else {
                const float s = scale_of(scale[i]);
                to[place(row, 2 * u)] = eight_of(v[i][0], v[i][1], s);
                to[place(row, 2 * u + 1)] = eight_of(v[i][2], v[i][3], s);
            }
        }
    }
};

template <Kind KIND, int RT>
__global__ void __launch_bounds__(512) linear4_rows_kernel(Linear4Args a)
{
    extern __shared__ __attribute__((aligned(16))) u32x4 lds[];
    constexpr uint32_t kTileVecs = 16 * RT * 16;              // a k tile of the rows, in 16 bytes
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t quarter = wave / kSlabs, li = lane & 15, lq = lane >> 4;
    const Group4& g = a.groups[group_of(a, lane)];
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
            u32x4 o[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) o[r] = tile[((r * 4 + j) * 4 + lq) * 16 + (li ^ (lq * 4 + j))];
#pragma unroll
            for (int n = 0; n < kNt; ++n) {
                const u32x4 wv = weights_of(wt[n], j);
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[n][r] = mfma(wv, o[r], acc[n][r]);
            }
        }
    };
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
        if (mine) x.ask_last(whole, K - whole * kTile4K);
        lds_barrier();
        if (mine) x.put(tiles);
        lds_barrier();
        if (mine) multiply(wl, tiles);
    }
    // quarter q finishes the tiles t with t % 4 = q of its slab, with the sums of the other quarters
    f32x4 bias[kNt * RT / kQuarters];
#pragma unroll
    for (int i = 0; i < kNt * RT / kQuarters; ++i) bias[i] = bias_of(a, g, (slab * kNt + (i * kQuarters + quarter) / RT) * kTile4Rows + 4 * lq);
    __syncthreads();
    f32x4* part = (f32x4*)lds;
    const auto at = [&](uint32_t q, uint32_t t) { return ((q * kSlabs + wave % kSlabs) * (kNt * RT) + t) * 64 + lane; };
#pragma unroll
    for (int t = 0; t < kNt * RT; ++t) if (t % kQuarters != (int)quarter) part[at(quarter, t)] = acc[t / RT][t % RT];
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kNt * RT; ++t) {
        if (t % kQuarters != (int)quarter) continue;
        f32x4 v = acc[t / RT][t % RT] + bias[t / kQuarters];
#pragma unroll
        for (int o = 1; o < kQuarters; ++o) v += part[at((quarter + o) % kQuarters, t)];
        finish_tile(a, g, (slab * kNt + t / RT) * kTile4Rows + 4 * lq, first_row + 16 * (t % RT) + li, v);
    }
}
template <int RT> constexpr uint32_t rows_lds() { return kQuarters * kSlabs * (kNt * RT) * 1024; }      // the sums at the end; both buffers of rows take no more
static_assert(rows_lds<4>() >= kQuarters * 2 * 64 * 256 && rows_lds<4>() <= 160 * 1024, "LDS");

template <Kind KIND, int RT, int NT, int DEPTH>
hipError_t go(const Linear4Args& a, uint32_t grid, hipStream_t s)
{
    hipLaunchKernelGGL((linear4_kernel<KIND, RT, NT, DEPTH>), dim3(grid), dim3(kWaves4 * 64), 0, s, a);
    return hipGetLastError();
}

template <Kind KIND, int RT>
hipError_t go_rows(const Linear4Args& a, uint32_t grid, hipStream_t s)
{
    hipLaunchKernelGGL((linear4_rows_kernel<KIND, RT>), dim3(grid), dim3(512), rows_lds<RT>(), s, a);
    return hipGetLastError();
}

template <Kind KIND>
hipError_t choose(const Linear4Args& a, Linear4Shape shape, uint32_t grid, hipStream_t s)
{
    if (shape.rt == 1) return shape.nt == 1 ? go<KIND, 1, 1, KIND == kRowsF32 ? 1 : 4>(a, grid, s) : go<KIND, 1, 4, 1>(a, grid, s);
    if constexpr (KIND == kRowsF32) return go<KIND, 2, 4, 1>(a, grid, s);
    else return shape.rt == 2 ? go_rows<KIND, 2>(a, grid, s) : go_rows<KIND, 4>(a, grid, s);
}

template <Kind KIND, int RT>
hipError_t prepare_rows() { return hipFuncSetAttribute((const void*)linear4_rows_kernel<KIND, RT>, hipFuncAttributeMaxDynamicSharedMemorySize, rows_lds<RT>()); }

}  // namespace

Linear4Shape linear4_shape(uint64_t tiles, uint32_t, uint32_t most_rows, uint32_t n_cus, uint32_t x_dtype)
{
    Linear4Shape s;
    s.rt = most_rows <= 16 ? 1 : most_rows <= 32 || x_dtype == MT_F32 ? 2 : 4;
    s.nt = s.rt > 1 ? (x_dtype == MT_F32 ? 4 : kNt * kSlabs) : tiles >= 16 * (uint64_t)n_cus ? 4 : 1;
    return s;
}

hipError_t prepare_linear4()
{
    hipError_t e = prepare_rows<kRowsBf16, 2>();
    if (e == hipSuccess) e = prepare_rows<kRowsBf16, 4>();
    if (e == hipSuccess) e = prepare_rows<kRowsMx8, 2>();
    return e == hipSuccess ? prepare_rows<kRowsMx8, 4>() : e;
}

hipError_t launch_linear4(const Linear4Args& a, Linear4Shape shape, uint32_t x_dtype, uint32_t grid, hipStream_t s)
{
    if (x_dtype == MT_MX8) return choose<kRowsMx8>(a, shape, grid, s);
    return x_dtype == MT_BF16 ? choose<kRowsBf16>(a, shape, grid, s) : choose<kRowsF32>(a, shape, grid, s);
}

}  // namespace mt
