// mt_attend: new tokens attend to all of their sequence's tokens in a paged cache.
//
// One pass over the cache with the running maximum m and sum l of a softmax: with S = scale q.k, p = 2^(log2(e) S - m), l = sum p, O = sum p v; where m grows, l and O
// are rescaled. out = O / l, lse = ln 2 (m + log2 l).
//
// Sixteen columns (query heads of one head of the cache, and with several new tokens these side by side) share what is loaded: S^T = K Q^T and O^T = V^T P^T on 16x16
// matrix instructions. A lane's 16 bytes of the cache are kEach values; a step is 4 kEach tokens. The rows of the first product are dealt so that the lane that gets a column's weights of kEach
// consecutive tokens is the one that needs them as operand of the second, whose other operand, the values feature by feature, is 16 bytes of memory as they lie: no weight
// and no value moves between lanes, and nothing goes through LDS before the end.
//
// A workgroup's four waves take steps in turn, each with sums of its own, joined in LDS. Long sequences are cut into parts of a workgroup each; the last of a tile's parts to
// end joins what all have left in the scratch.
//
// Bound by the cache's bytes, each fetched once. One new token, 128 elements a head: 64 requests of up to 4096 tokens, 8 bf16 heads of the cache, 119 us, 4.7 TB/s; one of 131072 tokens 103 us, 5.2;
// 32 of 12289 to 16384 in 8 bits 187 us, 5.1. One of 333 tokens, two heads of 64, is 5.6 us: a launch and a chain of four trips to memory. Two workgroups to a compute unit (eight waves, 256 registers each): a third
// spills (122 -> 183 us in the first of these). Loads that bypass the caches: 122 -> 145. fp32 rows run on fp32 matrix instructions, a sixteenth of the rate: over an 8-bit cache they, not memory, bound it (2.4 TB/s).
#include "lm_cache_device.h"

namespace mt {
namespace {

constexpr float kLowest = -3.402823466e38f, kNone = -__builtin_inff();
constexpr uint32_t kWaves = 4, kColumns = 16;
constexpr uint32_t kTickets = 4096;               // most tiles of a call that is cut into parts
constexpr uint32_t kRecords = 8192;               // most parts of a call
constexpr uint32_t kMaxParts = 64;                // ... of a tile
constexpr uint32_t kAhead = 16;
constexpr float kSlack = 8.0f;                    // m may lag behind by this: weights up to 2^8 are as exact as those up to 1

inline __host__ __device__ uint32_t record_floats(uint32_t dim) { return kColumns * (dim + 2); }

// How a call is cut.
struct Cut {
    uint32_t tiles;              // of a sequence and head
    uint32_t parts, part_len;    // most parts of a tile; tokens of one
};

struct AttendCall {
    AttendArgs g;
    Cut cut;
    uint32_t page_shift;
};

__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(float a, float b, const f32x4& acc) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, acc, 0, 0, 0); }

// Eight e4m3 values as bf16.
__device__ __forceinline__ u32x4 eight_bf16(uint32_t a, uint32_t b)
{
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true))};
}
__device__ __forceinline__ float e4m3_of(uint32_t w, int i)
{
    return i == 0 ? __builtin_amdgcn_cvt_f32_fp8(w, 0) : i == 1 ? __builtin_amdgcn_cvt_f32_fp8(w, 1) : i == 2 ? __builtin_amdgcn_cvt_f32_fp8(w, 2) : __builtin_amdgcn_cvt_f32_fp8(w, 3);
}

// Over the four lanes that hold a column.
template <typename F> __device__ __forceinline__ float over_column(float v, F f)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    v = f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    const uint32_t c = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane16_swap(c, c, false, false);
    return f(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
}

// Products of sixteen tokens' keys with the columns' queries, of sixteen elements' values with the columns' weights.  T: type of rows, C: of the cache.  D: a head's elements, or
// with EXACT false the most.
template <typename T, typename C, int D, bool EXACT> struct Shape {
    static constexpr int kEach = 16 / sizeof(C), kStep = 4 * kEach, kTiles = kEach / 4;
    static constexpr int kChunks = (D + 4 * kEach - 1) / (4 * kEach);       // loads of 16 bytes a lane for sixteen tokens' keys
    static constexpr int kDims = D / 16;
    static constexpr bool kNarrow = sizeof(C) == 1, kWide = sizeof(T) == 4;
    static constexpr int kQueries = kChunks * (kWide ? kEach / 4 : kEach / 8);       // 16-byte registers of a lane's queries

    // Elements of a head that chunk u of a lane has: kEach from here on.
    static __device__ __forceinline__ int first_of(int u, int g) { return 4 * kEach * u + kEach * g; }

    static __device__ __forceinline__ void load_queries(u32x4 (&q)[kQueries], const T* row, int g, uint32_t dim, bool there)
    {
        constexpr int per = 16 / sizeof(T);
#pragma unroll
        for (int u = 0; u < kChunks; ++u)
#pragma unroll
            for (int e = 0; e < kEach / per; ++e) {
                const uint32_t at = first_of(u, g) + per * e;
                u32x4 v{0, 0, 0, 0};
                if (there && at < (EXACT ? D : dim)) v = *(const typename Any<T>::vec16*)(row + at);
                q[u * (kEach / per) + e] = v;
            }
    }

    static __device__ __forceinline__ f32x4 scores(const u32x4 (&k)[kChunks], const u32x4 (&q)[kQueries])
    {
        f32x4 s{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
            if constexpr (kWide) {
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const float a = kNarrow ? e4m3_of(k[u][e / 4], e % 4) : __builtin_bit_cast(f32x4, k[u])[e % 4];
                    s = mfma(a, __builtin_bit_cast(f32x4, q[u * (kEach / 4) + e / 4])[e % 4], s);
                }
            } else if constexpr (kNarrow) {
                s = mfma(eight_bf16(k[u][0], k[u][1]), q[2 * u], s);
                s = mfma(eight_bf16(k[u][2], k[u][3]), q[2 * u + 1], s);
            } else s = mfma(k[u], q[u], s);
        }
        return s;
    }

    // p: the weights as the second product takes them.
    static constexpr int kWeights = kWide ? kEach : kEach / 8;
    struct Weights {
        u32x4 v[kWide ? 1 : kEach / 8], rest[kWide ? 1 : kEach / 8];       // a weight's first bf16 bits, cut off, and the next, rounded: together up to 2^-16 of it off
        float f[kWide ? kEach : 1];
    };
    // (never 0 for a weight that isn't: an infinite value times either part is the same infinity. 2^-40 of it is far below what the sum shows)
    static __device__ __forceinline__ float rest_of(float p) { return fmaf(p, 9.094947e-13f, p - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, p) & 0xffff0000u)); }
    static __device__ __forceinline__ Weights weights(const float (&p)[kEach])
    {
        Weights w{};
        if constexpr (kWide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) w.f[e] = p[e];
        } else {
#pragma unroll
            for (int e = 0; e < kEach / 2; ++e) {
                const uint32_t a = __builtin_bit_cast(uint32_t, p[2 * e]), b = __builtin_bit_cast(uint32_t, p[2 * e + 1]);
                w.v[e / 4][e % 4] = __builtin_amdgcn_perm(b, a, 0x07060302u);        // the upper halves
                w.rest[e / 4][e % 4] = pack_bf16(rest_of(p[2 * e]), rest_of(p[2 * e + 1]));
            }
        }
        return w;
    }
    static __device__ __forceinline__ f32x4 add_values(const u32x4& v, const Weights& w, f32x4 o)
    {
        if constexpr (kWide) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) o = mfma(kNarrow ? e4m3_of(v[e / 4], e % 4) : __builtin_bit_cast(f32x4, v)[e % 4], w.f[e], o);
        } else if constexpr (kNarrow) {
            const u32x4 a = eight_bf16(v[0], v[1]), b = eight_bf16(v[2], v[3]);
            o = mfma(a, w.rest[0], o);
            o = mfma(b, w.rest[1], o);
            o = mfma(a, w.v[0], o);
            o = mfma(b, w.v[1], o);
        } else {
            o = mfma(v, w.rest[0], o);
            o = mfma(v, w.v[0], o);
        }
        return o;
    }

    // v with the elements outside of first .. last - 1 zeroed.
    static __device__ __forceinline__ u32x4 only(u32x4 v, int first, int last)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t keep = 0;
#pragma unroll
            for (int b = 0; b < 4; b += sizeof(C)) {
                const int e = (4 * i + b) / (int)sizeof(C);
                keep |= e >= first && e < last ? (sizeof(C) == 4 ? 0xffffffffu : ((1u << 8 * (sizeof(C) % 4)) - 1) << 8 * b) : 0;
            }
            v[i] &= keep;
        }
        return v;
    }
    // Whether an element is infinite or NaN.
    static __device__ __forceinline__ bool odd(const u32x4& v)
    {
        bool r = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(C) == 4) r |= (v[i] & 0x7f800000u) == 0x7f800000u;
            else if constexpr (sizeof(C) == 2) r |= (v[i] & 0x7f800000u) == 0x7f800000u || (v[i] & 0x7f80u) == 0x7f80u;
            else
#pragma unroll
                for (int b = 0; b < 32; b += 8) r |= (v[i] >> b & 0x7fu) == 0x7fu;
        }
        return r;
    }
};

__device__ __forceinline__ void hand_over(float* p, float a, float b)
{
    __hip_atomic_store((uint64_t*)p, (uint64_t)__builtin_bit_cast(uint32_t, a) | (uint64_t)__builtin_bit_cast(uint32_t, b) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
struct Two { float a, b; };
__device__ __forceinline__ Two take_over(const float* p)
{
    const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return Two{__builtin_bit_cast(float, (uint32_t)v), __builtin_bit_cast(float, (uint32_t)(v >> 32))};
}

// 16 lanes' worth of a factor: 2^(a - b), 0 where a is nothing yet.
__device__ __forceinline__ float factor(float m, float to) { return __builtin_amdgcn_exp2f(m - to); }

// MANY: columns are (new token, query head) pairs of one head; else the query heads of one row.
template <typename T, typename C, int D, bool EXACT, bool MANY>
__global__ void __launch_bounds__(64 * kWaves, D > 128 || (sizeof(T) == 4 && sizeof(C) == 1 && MANY) ? 1 : 2) attend_kernel(AttendCall call)
{
    using S = Shape<T, C, D, EXACT>;
    constexpr int kEach = S::kEach, kStep = S::kStep, kTiles = S::kTiles;
    const mt_kv_cache& c = call.g.c;
    const mt_attend_args& a = call.g.a;
    constexpr int kRow = D + 4;
    constexpr uint32_t kPlanes = D > 128 ? 2 : kWaves;            // (64 KiB of LDS)
    __shared__ __attribute__((aligned(16))) float sums[kPlanes][kColumns][kRow];
    __shared__ float wave_m[kWaves][kColumns], wave_l[kWaves][kColumns], col_m[kColumns], col_l[kColumns];
    __shared__ float part_m[kMaxParts][kColumns], part_l[kMaxParts][kColumns];
    __shared__ uint32_t last_part;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const uint32_t dim = EXACT ? D : c.head_dim, G = a.q_heads / c.heads;
    // workgroups of one sequence and head lie eight apart, on one XCD
    const uint32_t pairs = call.g.b.n_seqs * c.heads, tiles = call.cut.tiles, eights = pairs / 8 * 8 * tiles;
    uint32_t pair, tile;
    if (blockIdx.x < eights) { const uint32_t at = blockIdx.x / 8; pair = at / tiles * 8 + blockIdx.x % 8; tile = at % tiles; }
    else { const uint32_t at = blockIdx.x - eights, left = pairs % 8; pair = pairs / 8 * 8 + at % left; tile = at / left; }
    const uint32_t entry = pair / c.heads, h = pair % c.heads, part = gridDim.y - 1 - blockIdx.y;      // (ends of long sequences first, short sequences last)
    const SeqRows s = seq_rows(c, call.g.b, entry);
    const uint32_t rows = (uint32_t)max(s.last - s.first, 0), head_tiles = (G + kColumns - 1) / kColumns;
    const uint32_t all_tiles = MANY ? (rows * G + kColumns - 1) / kColumns : rows * head_tiles;        // (rows * G is below 2^31)
    const int32_t reach = (int32_t)min((uint32_t)s.length, c.table_width << call.page_shift);
    const int32_t* table = c.table + (uint64_t)max(s.seq, 0) * c.table_stride;
    const uint64_t at_head = a.layer * c.layer_stride + (uint64_t)h * c.page_tokens * dim;
    const C *keys = (const C*)c.k + at_head, *values = (const C*)c.v + at_head;
    const uint64_t at_scales = S::kNarrow ? a.layer * c.scales_layer_stride + h * c.page_tokens : 0;
    const float to_log2 = a.scale * 1.44269504f;

    // Pages of this lane's tokens of a step: kEach from kEach (n / 4) on for its keys, from kEach g on for everything else.  Entries behind the sequence's are read, and not used.
    const int32_t stride = kWaves * kStep, k_at = kEach * (n >> 2), v_at = kEach * g, last_entry = (int32_t)c.table_width - 1;
    const auto page_at = [&](int32_t token) { return table[min(token >> call.page_shift, last_entry)]; };

    for (uint32_t t = tile; t < all_tiles; t += tiles) {
        // tiles beyond those that the call has reckoned with are not cut
        const bool planned = t < tiles;
        if (!planned && part > 0) break;
        // this lane's column: its row, its query head, the tokens that it sees
        const uint32_t first_col = MANY ? t * kColumns : t % head_tiles * kColumns, row0 = MANY ? 0 : t / head_tiles;
        const uint32_t col = first_col + n, j = MANY ? col / G : row0, hg = MANY ? col % G : col;
        const bool there = MANY ? j < rows : col < G;
        const auto end_of = [&](uint32_t r) { return min(max(s.upto((int32_t)r), 0), reach); };
        const auto begin_of = [&](uint32_t r) {
            const int32_t upto = s.upto((int32_t)r);
            return a.window && upto > 0 && a.window < (uint32_t)upto ? min(upto - (int32_t)a.window, reach) : 0;
        };
        const uint32_t top_row = MANY ? first_col / G : row0, bottom_row = MANY ? min((first_col + kColumns - 1) / G, rows - 1) : row0;
        const int32_t lo = begin_of(top_row), hi = end_of(bottom_row);              // what some column sees,
        const int32_t all_lo = begin_of(bottom_row), all_hi = end_of(top_row);      // what all see
        const int32_t mine_lo = there ? begin_of(j) : lo, mine_hi = there ? end_of(j) : hi;

        const int32_t start = lo / 64 * 64;
        const uint32_t parts = hi <= lo || !planned ? 1 : min(((uint32_t)(hi - start) + call.cut.part_len - 1) / call.cut.part_len, call.cut.parts);
        if (part >= parts) break;
        const int32_t from = start + (int32_t)(part * call.cut.part_len), to = part + 1 == parts ? hi : from + (int32_t)call.cut.part_len;

        const T* row = (const T*)a.q + (there ? (uint64_t)((uint32_t)s.first + j) * a.q_stride + ((uint64_t)h * G + hg) * dim : 0);
        u32x4 q[S::kQueries];
        S::load_queries(q, row, g, dim, there);

        f32x4 o[S::kDims];
#pragma unroll
        for (int d = 0; d < S::kDims; ++d) o[d] = f32x4{0, 0, 0, 0};
        float m = kLowest, l = 0;

        const auto usable = [&](int32_t page, int32_t token) { return token < to && (uint32_t)page < c.n_pages; };
        const uint32_t in_page = c.page_tokens - 1;
        const auto load_keys = [&](u32x4 (&k)[kTiles][S::kChunks], int32_t page, int32_t token) {
            const C* p = keys + (usable(page, token) ? (uint32_t)page : 0) * c.page_stride + (((uint32_t)token & in_page) + (n & 3)) * dim;
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int u = 0; u < S::kChunks; ++u) {
                    const uint32_t at = S::first_of(u, g);
                    if constexpr (EXACT && D % (4 * kEach) == 0) k[i][u] = *(const u32x4*)(p + 4 * i * dim + at);
                    else {
                        k[i][u] = *(const u32x4*)(p + 4 * i * dim + (at < dim ? at : 0));
                        if (at >= dim) k[i][u] = u32x4{0, 0, 0, 0};
                    }
                }
        };
        int32_t token = from + (int32_t)wave * kStep;
        if (token < to) {
            u32x4 k[kTiles][S::kChunks];
            int32_t k_page = page_at(token + k_at), v_page = page_at(token + v_at);
            int32_t next_k = page_at(token + stride + k_at), next_v = page_at(token + stride + v_at);
            load_keys(k, k_page, token + k_at);
            for (; token < to; token += stride) {
                // values and scales of this step, the pages of the one behind the next
                const bool v_there = usable(v_page, token + v_at);
                const uint32_t slot = (uint32_t)(token + v_at) & in_page, vp = v_there ? (uint32_t)v_page : 0;
                const C* p = values + vp * c.page_stride + (uint32_t)n * c.page_tokens + slot;
                u32x4 v[S::kDims], ks, vs;
#pragma unroll
                for (int d = 0; d < S::kDims; ++d) v[d] = *(const u32x4*)(p + (EXACT || 16u * d < dim ? 16 * d * c.page_tokens : 0));
                if constexpr (S::kNarrow) {
                    ks = *(const u32x4*)(c.k_scales + at_scales + vp * c.scales_page_stride + slot);
                    vs = *(const u32x4*)(c.v_scales + at_scales + vp * c.scales_page_stride + slot);
                }
                const int32_t after_k = page_at(token + 2 * stride + k_at), after_v = page_at(token + 2 * stride + v_at);
                float x[kEach];
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    const f32x4 sc = S::scores(k[i], q);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[4 * i + e] = sc[e] * to_log2;
                }
                // (behind the last step: this one's again, from the caches)
                const bool more = token + stride < to;
                load_keys(k, more ? next_k : k_page, (more ? token + stride : token) + k_at);
                if constexpr (S::kNarrow)
#pragma unroll
                    for (int e = 0; e < kEach; ++e) x[e] *= of_scale(ks[e / 4] >> 8 * (e % 4) & 255);
                const bool whole = token >= all_lo && token + kStep <= min(all_hi, to) && !__ballot(!v_there);
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < kEach; ++e) {
                        const int32_t at = token + v_at + e;
                        if (!(v_there && at >= mine_lo && at < min(mine_hi, to))) x[e] = kNone;
                    }
                }
                float most = x[0];
#pragma unroll
                for (int e = 1; e < kEach; ++e) most = fmaxf(most, x[e]);
                most = over_column(most, [](float p, float q) { return fmaxf(p, q); });
                if (__ballot(most > m + kSlack)) {
                    // (never infinite: a product of +infinity has an infinite weight then, and so l, where infinity less infinity would say NaN)
                    const float grown = most > m + kSlack ? fminf(most, -kLowest) : m, f = factor(m, grown);
                    m = grown;
                    l *= f;
#pragma unroll
                    for (int d = 0; d < S::kDims; ++d) o[d] *= f;
                }
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    x[e] = __builtin_amdgcn_exp2f(x[e] - m);
                    l += x[e];
                }
                if constexpr (S::kNarrow)
#pragma unroll
                    for (int e = 0; e < kEach; ++e) x[e] *= of_scale(vs[e / 4] >> 8 * (e % 4) & 255);
                if (!whole) {
                    // what no column sees counts nothing, whatever stands there
                    const int first = lo - (token + v_at), last = v_there ? min(hi, to) - (token + v_at) : 0;
                    bool odd = false;
#pragma unroll
                    for (int e = 0; e < kEach; ++e) {
                        const int32_t at = token + v_at + e;
                        if (!(v_there && at >= mine_lo && at < min(mine_hi, to))) x[e] = 0;
                    }
#pragma unroll
                    for (int d = 0; d < S::kDims; ++d) {
                        v[d] = S::only(v[d], first, last);
                        if constexpr (MANY) odd |= S::odd(v[d]);
                    }
                    if (MANY && __ballot(odd)) {
                        // infinities or NaN among values that some columns see and others don't: token by token, each for the columns that see it
#pragma nounroll
                        for (int i = 0; i < kStep; ++i) {
                            const typename S::Weights w = S::weights(x);
                            const bool sees = token + i >= mine_lo && token + i < min(mine_hi, to);
#pragma unroll
                            for (int d = 0; d < S::kDims; ++d) {
                                const f32x4 with = S::add_values(S::only(v[d], i - v_at, i - v_at + 1), w, o[d]);
                                if (sees) o[d] = with;
                            }
                        }
#pragma unroll
                        for (int d = 0; d < S::kDims; ++d) v[d] = u32x4{0, 0, 0, 0};
                    }
                }
                const typename S::Weights w = S::weights(x);
#pragma unroll
                for (int d = 0; d < S::kDims; ++d)
                    if (EXACT || 16u * d < dim) o[d] = S::add_values(v[d], w, o[d]);
                k_page = next_k; v_page = next_v;
                next_k = after_k; next_v = after_v;
            }
        }
        l = over_column(l, [](float p, float q) { return p + q; });

        // the waves' sums, one after the other's statistics
        __syncthreads();
        if (g == 0) { wave_m[wave][n] = m; wave_l[wave][n] = l; }
        __syncthreads();
        float top = wave_m[0][n];
#pragma unroll
        for (uint32_t w = 1; w < kWaves; ++w) top = fmaxf(top, wave_m[w][n]);
        const float f = factor(m, top);
#pragma unroll
        for (uint32_t plane = 0; plane < kWaves; plane += kPlanes) {
            if (plane) __syncthreads();
            if (wave >= plane && wave < plane + kPlanes)
#pragma unroll
                for (int d = 0; d < S::kDims; ++d)
                    if (EXACT || 16u * d < dim) {
                        f32x4* to = (f32x4*)&sums[wave - plane][n][16 * d + 4 * g];
                        *to = plane ? *to + o[d] * f : o[d] * f;
                    }
        }
        if (wave == 0 && g == 0) {
            float total = 0;
#pragma unroll
            for (uint32_t w = 0; w < kWaves; ++w) total += wave_l[w][n] * factor(wave_m[w][n], top);
            col_m[n] = top; col_l[n] = total;
        }
        __syncthreads();
        const uint32_t cols = min((MANY ? rows * G : G) - first_col, kColumns);
        float* records = (float*)((uint8_t*)a.scratch + kTickets * 4);
        const uint32_t tile_at = pair * tiles + t, half = dim / 2;
        if (parts > 1) {
            float* mine = records + ((uint64_t)tile_at * call.cut.parts + part) * record_floats(dim);
            for (uint32_t i = threadIdx.x; i < cols * half; i += 64 * kWaves) {
                const uint32_t cc = i / half, d = i % half * 2;
                float p = 0, r = 0;
#pragma unroll
                for (uint32_t w = 0; w < kPlanes; ++w) { p += sums[w][cc][d]; r += sums[w][cc][d + 1]; }
                hand_over(mine + 2 * kColumns + cc * dim + d, p, r);
            }
            if (threadIdx.x < cols) hand_over(mine + 2 * threadIdx.x, col_m[threadIdx.x], col_l[threadIdx.x]);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0) last_part = __hip_atomic_fetch_add((uint32_t*)a.scratch + tile_at, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
            __syncthreads();
            if (!last_part) continue;
            if (threadIdx.x == 0) __hip_atomic_store((uint32_t*)a.scratch + tile_at, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // ready for the next call
            // statistics of all parts, a thread to a part and column; then a thread to two elements, kAhead parts on their way at a time (the first of them with the statistics)
            const float* all = records + (uint64_t)tile_at * call.cut.parts * record_floats(dim);
            const auto load_some = [&](Two (&v)[kAhead], uint32_t i, uint32_t k) {
                const float* one = all + 2 * kColumns + i / half * dim + i % half * 2;
#pragma unroll
                for (uint32_t e = 0; e < kAhead; ++e) v[e] = take_over(one + (uint64_t)min(k + e, parts - 1) * record_floats(dim));
            };
            Two v[kAhead];
            for (uint32_t i = threadIdx.x; i < parts * kColumns; i += 64 * kWaves) {
                const uint32_t cc = i % kColumns;
                const Two r = cc < cols ? take_over(all + (uint64_t)(i / kColumns) * record_floats(dim) + 2 * cc) : Two{kLowest, 0};
                part_m[i / kColumns][cc] = r.a; part_l[i / kColumns][cc] = r.b;
            }
            __syncthreads();
            if (threadIdx.x < kColumns) {
                float top = kLowest, total = 0;
                for (uint32_t i = 0; i < parts; ++i) top = fmaxf(top, part_m[i][threadIdx.x]);
                for (uint32_t i = 0; i < parts; ++i) {
                    const float f = factor(part_m[i][threadIdx.x], top);
                    total += part_l[i][threadIdx.x] * f;
                    part_m[i][threadIdx.x] = f;
                }
                col_m[threadIdx.x] = top; col_l[threadIdx.x] = total;
            }
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < cols * half; i += 64 * kWaves) {
                const uint32_t cc = i / half, d = i % half * 2;
                float p = 0, r = 0;
                for (uint32_t k = 0; k < parts; k += kAhead) {
                    load_some(v, i, k);
#pragma unroll
                    for (uint32_t e = 0; e < kAhead; ++e) {
                        // (loads behind the last part have read it again: left out, not multiplied by 0, which an infinite sum would make NaN)
                        if (k + e >= parts) break;
                        const float f = part_m[k + e][cc];
                        p = fmaf(v[e].a, f, p); r = fmaf(v[e].b, f, r);
                    }
                }
                sums[0][cc][d] = p; sums[0][cc][d + 1] = r;
            }
            __syncthreads();
        }
        for (uint32_t i = threadIdx.x; i < cols * dim; i += 64 * kWaves) {
            const uint32_t cc = i / dim, d = i % dim;
            const uint32_t out_col = first_col + cc, out_row = (uint32_t)s.first + (MANY ? out_col / G : row0), out_head = h * G + (MANY ? out_col % G : out_col);
            float sum = sums[0][cc][d];
            if (parts == 1)
#pragma unroll
                for (uint32_t w = 1; w < kPlanes; ++w) sum += sums[w][cc][d];
            const float total = col_l[cc];
            ((T*)a.out)[(uint64_t)out_row * a.out_stride + (uint64_t)out_head * dim + d] = (T)(total == 0.0f ? 0.0f : sum / total);
            if (d == 0 && a.lse) a.lse[(uint64_t)out_row * a.q_heads + out_head] = total == 0.0f ? kNone : (col_m[cc] + log2f(total)) * 0.693147181f;
        }
    }
}

// Tiles of a sequence and head, and how many parts a tile of the longest sequence is cut into.
// Parts wanted of a call, 512 / 1024 / 2048 / 4096: 64 requests of up to 4096 tokens bf16 139 / 132 / 122 / 126 us, 32 of 12289 to 16384 in 8 bits 179 / 183 / 183 / 190. Parts of a tile at most, 64 / 128:
// one request of 131072 103 / 115 (the join reads them one after another). Tokens of a part at least, 64 / 128 / 256 / 512 / 1024: one request of 2000 tokens in 8 bits 12.8 / 10.8 / 11.5 / 14.0 / 18.7,
// one of 8000 bf16 21.8 / 21.6 / 16.2 / 16.0 / 22.0, 16 of 100 to 1500 22.1 / 21.8 / 17.7 / 22.6 / 22.1. Not cut up to 512 tokens: 333 tokens whole 5.9 us, in two parts 7.5; 700 tokens 14.9 and 11.2.
constexpr uint64_t kLeast = 256, kWhole = 512, kPartUnit = 256, kWanted = 2048;
uint64_t most_parts(uint64_t tiles)
{
    return tiles > kTickets ? 1 : std::min<uint64_t>(std::min<uint64_t>(std::max<uint64_t>(kWanted / tiles, 1), kRecords / tiles), kMaxParts);
}
Cut cut_of(const mt_kv_cache& c, const mt_kv_batch& b, uint32_t q_heads, uint32_t max_length, uint32_t window)
{
    // (tiles and tokens beyond these are the kernel's loops')
    constexpr uint64_t most_new = 1u << 16, most_tiles = 1u << 22;
    const uint64_t G = q_heads / c.heads, new_rows = std::min<uint64_t>(b.max_new, most_new), pairs = (uint64_t)b.n_seqs * c.heads;
    const uint64_t each = new_rows > 1 ? (new_rows * G + kColumns - 1) / kColumns : (G + kColumns - 1) / kColumns;
    Cut cut{(uint32_t)std::min<uint64_t>(each, std::max<uint64_t>(most_tiles / pairs, 1)), 1, 0};
    const uint64_t reach = (uint64_t)c.table_width * c.page_tokens;
    uint64_t longest = max_length ? std::min<uint64_t>(max_length, reach) : reach;
    if (window) longest = std::min<uint64_t>(longest, (uint64_t)window + new_rows + 64);
    const uint64_t parts = longest <= kWhole ? 1 : most_parts(pairs * cut.tiles), len = std::max<uint64_t>(kLeast, ((std::max<uint64_t>(longest, 1) + parts - 1) / parts + kPartUnit - 1) / kPartUnit * kPartUnit);
    cut.part_len = (uint32_t)len;
    cut.parts = (uint32_t)((longest + len - 1) / len);
    return cut;
}

template <typename T, typename C, int D, bool EXACT>
hipError_t go(const AttendCall& call, hipStream_t s)
{
    const dim3 grid(call.g.b.n_seqs * call.g.c.heads * call.cut.tiles, call.cut.parts);
    return launch(call.g.b.max_new > 1 ? attend_kernel<T, C, D, EXACT, true> : attend_kernel<T, C, D, EXACT, false>, grid, 64 * kWaves, 0, s, call);
}
template <typename T, typename C>
hipError_t choose(const AttendCall& call, hipStream_t s)
{
    const uint32_t dim = call.g.c.head_dim;
    if (dim == 64) return go<T, C, 64, true>(call, s);
    if (dim == 128) return go<T, C, 128, true>(call, s);
    return dim < 128 ? go<T, C, 128, false>(call, s) : go<T, C, 256, false>(call, s);
}

}  // namespace

uint64_t attend_scratch_bytes(const mt_kv_cache& c, const mt_kv_batch& b, uint32_t q_heads, uint32_t max_length)
{
    // (what suffices for any window and any shorter longest sequence)
    const uint64_t tiles = (uint64_t)b.n_seqs * c.heads * cut_of(c, b, q_heads, 0, 0).tiles, reach = (uint64_t)c.table_width * c.page_tokens;
    const uint64_t parts = std::min(most_parts(tiles), ((max_length ? std::min<uint64_t>(max_length, reach) : reach) + kLeast - 1) / kLeast);
    return parts > 1 ? kTickets * 4 + tiles * parts * record_floats(c.head_dim) * 4 : 0;
}

hipError_t launch_attend(const AttendArgs& g, hipStream_t s)
{
    AttendCall call{g, cut_of(g.c, g.b, g.a.q_heads, g.a.max_length, g.a.window), 4};
    while ((1u << call.page_shift) < g.c.page_tokens) ++call.page_shift;
    const bool narrow = g.c.dtype == MT_KV8;
    if (g.a.dtype == MT_BF16) return narrow ? choose<__bf16, uint8_t>(call, s) : choose<__bf16, __bf16>(call, s);
    return narrow ? choose<float, uint8_t>(call, s) : choose<float, float>(call, s);
}

}  // namespace mt
