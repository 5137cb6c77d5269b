// mt_kv_write: new tokens' keys and values into their pages.
//
// A token's keys lie side by side, its values page_tokens apart; in 8 bits a token and head share the power of two that the largest magnitude takes. A few tokens of a sequence: a wave to a token and head,
// its values scattered element by element (256 sequences of one token, eight heads of 128, in 8 bits: 6.3 us, a chain of three trips to memory). Many: a workgroup to a head and 64 places side by
// side, values turned around in LDS and written 16 bytes of a feature at a time (eight prompts of 1500 to 4096 tokens, eight heads of 128 bf16 elements: 58.6 us, 4.1 TB/s; into 8 bits 56, 3.2; pairs of elements to a lane, half of the
// loads on their way: 107).
#include <type_traits>

#include "lm_cache_device.h"

namespace mt {
namespace {

// Two consecutive elements, as they come and as values.
template <typename T> struct Pair;
template <> struct Pair<__bf16> {
    typedef uint32_t raw __attribute__((aligned(2)));
    static __device__ __forceinline__ float lo(uint32_t v) { return bf16_lo(v); }
    static __device__ __forceinline__ float hi(uint32_t v) { return bf16_hi(v); }
};
template <> struct Pair<float> {
    typedef u32x2 raw __attribute__((aligned(4)));
    static __device__ __forceinline__ float lo(const u32x2& v) { return __builtin_bit_cast(float, (uint32_t)v[0]); }
    static __device__ __forceinline__ float hi(const u32x2& v) { return __builtin_bit_cast(float, (uint32_t)v[1]); }
};
template <typename T> using RawPair = std::remove_cv_t<std::conditional_t<sizeof(T) == 2, uint32_t, u32x2>>;

// A wave's elements of one head of a token: lane l has elements 2 l and 2 l + 1, and 128 on.
template <typename T> struct HeadOf {
    static constexpr uint32_t kPairs = MT_KV_MAX_DIM / 128;
    RawPair<T> v[kPairs];
    __device__ __forceinline__ void load(const T* p, uint32_t lane, uint32_t dim)
    {
#pragma unroll
        for (uint32_t i = 0; i < kPairs; ++i) {
            v[i] = RawPair<T>{};
            if (128 * i + 2 * lane < dim) v[i] = *(const typename Pair<T>::raw*)(p + 128 * i + 2 * lane);
        }
    }
    // e8m0 of the largest magnitude, 255 with an infinity or NaN among them
    __device__ __forceinline__ uint32_t scale() const
    {
        float most = 0;
        bool odd = false;
#pragma unroll
        for (uint32_t i = 0; i < kPairs; ++i) {
            const float a = Pair<T>::lo(v[i]), b = Pair<T>::hi(v[i]);
            odd |= a != a || b != b;
            most = fmaxf(most, fmaxf(fabsf(a), fabsf(b)));
        }
        return __ballot(odd) ? 255 : scale_for(wave_max(most));
    }
    __device__ __forceinline__ uint32_t narrow(uint32_t i, float to) const { return two_e4m3(Pair<T>::lo(v[i]) * to, Pair<T>::hi(v[i]) * to); }
};

template <typename T, typename C>
__global__ void __launch_bounds__(256) kv_write_kernel(KvWriteArgs w)
{
    const mt_kv_cache& c = w.c;
    const uint32_t lane = threadIdx.x & 63, h = blockIdx.z * 4 + (threadIdx.x >> 6), D = c.head_dim;
    if (h >= c.heads) return;
    const SeqRows s = seq_rows(c, w.b, blockIdx.x);
    for (uint32_t j = blockIdx.y; (int32_t)j < s.last - s.first; j += gridDim.y) {
        const int64_t r = s.first + (int32_t)j;
        HeadOf<T> k, v;
        k.load((const T*)w.a.k + r * w.a.k_stride + h * D, lane, D);
        v.load((const T*)w.a.v + r * w.a.v_stride + h * D, lane, D);
        const int32_t token = s.upto((int32_t)j) - 1, page = s.seq < 0 ? -1 : page_of(c, s.seq, token);
        if (page < 0) continue;
        const uint32_t slot = (uint32_t)token % c.page_tokens;
        const uint64_t at = w.a.layer * c.layer_stride + page * c.page_stride + (uint64_t)h * c.page_tokens * D;
        C *ko = (C*)c.k + at + slot * D, *vo = (C*)c.v + at + slot;
        const uint32_t ke = sizeof(C) == 1 ? k.scale() : 0, ve = sizeof(C) == 1 ? v.scale() : 0;
        const float kf = to_scale(ke), vf = to_scale(ve);
#pragma unroll
        for (uint32_t i = 0; i < HeadOf<T>::kPairs; ++i) {
            const uint32_t d = 128 * i + 2 * lane;
            if (d >= D) continue;
            if constexpr (sizeof(C) == 1) {
                *(uint16_t*)(ko + d) = (uint16_t)k.narrow(i, kf);
                const uint32_t two = v.narrow(i, vf);
                vo[(uint64_t)d * c.page_tokens] = (uint8_t)two;
                vo[(uint64_t)(d + 1) * c.page_tokens] = (uint8_t)(two >> 8);
            } else {
                *(RawPair<T>*)(ko + d) = k.v[i];
                vo[(uint64_t)d * c.page_tokens] = (C)Pair<T>::lo(v.v[i]);
                vo[(uint64_t)(d + 1) * c.page_tokens] = (C)Pair<T>::hi(v.v[i]);
            }
        }
        if constexpr (sizeof(C) == 1) {
            const uint64_t to = w.a.layer * c.scales_layer_stride + page * c.scales_page_stride + h * c.page_tokens + slot;
            if (lane == 0) { c.k_scales[to] = (uint8_t)ke; c.v_scales[to] = (uint8_t)ve; }
        }
    }
}

// 64 places of a sequence and head (32 of fp32), eight elements to a thread at a time: keys go out as they come in, values wait in LDS for all of the places.
template <typename C> constexpr uint32_t places_of() { return sizeof(C) == 4 ? 32 : 64; }
template <typename T> struct Eight {
    u32x4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) v[i] = *(const typename Any<T>::vec16*)(p + 8 / (sizeof(T) / 2) * i);
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 2) return i % 2 ? bf16_hi(v[0][i / 2]) : bf16_lo(v[0][i / 2]);
        else return __builtin_bit_cast(f32x4, v[i / 4])[i % 4];
    }
    // The largest magnitude's bits; above infinity's with a NaN.
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, at(i)) & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ u32x2 narrow(float to) const
    {
        u32x2 r;
#pragma unroll
        for (int i = 0; i < 2; ++i) r[i] = two_e4m3(at(4 * i) * to, at(4 * i + 1) * to) | two_e4m3(at(4 * i + 2) * to, at(4 * i + 3) * to) << 16;
        return r;
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) *(u32x4*)(p + 8 / (sizeof(T) / 2) * i) = v[i];
    }
};

template <typename T, typename C>
__global__ void __launch_bounds__(256) kv_write_many_kernel(KvWriteArgs w)
{
    constexpr uint32_t kPlaces = places_of<C>(), kEach = 16 / sizeof(C), kAhead = 4, kPad = sizeof(C) == 4 ? 4 : 8;
    constexpr bool kNarrow = sizeof(C) == 1;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ uint32_t most[2][kPlaces];
    __shared__ int32_t pages[kPlaces / 16];
    const mt_kv_cache& c = w.c;
    const uint32_t tid = threadIdx.x, D = c.head_dim, row = D + kPad, eights = D / 8, pieces = kPlaces * eights;
    const uint32_t entry = blockIdx.x / c.heads, h = blockIdx.x % c.heads;
    C* tile = (C*)lds;                            // [kPlaces][row]
    const SeqRows s = seq_rows(c, w.b, entry);
    if (s.seq < 0 || s.last <= s.first) return;
    const Places rows = places_of_rows(s.length, s.first, s.last, s.after, (int32_t)(c.table_width * c.page_tokens));
    const int32_t begin = rows.begin, stop = rows.stop;
    const int64_t row0 = (int64_t)s.first - (s.upto(0) - 1);      // (row of place 0)
    const T *k_rows = (const T*)w.a.k + h * D, *v_rows = (const T*)w.a.v + h * D;
    for (int32_t group = begin / (int32_t)kPlaces + (int32_t)blockIdx.y; group * (int32_t)kPlaces < stop; group += (int32_t)gridDim.y) {
        const int32_t base = group * (int32_t)kPlaces, lo = max(begin - base, 0), hi = min(stop - base, (int32_t)kPlaces);
        if (tid < kPlaces / 16) pages[tid] = page_of(c, s.seq, base + 16 * (int32_t)tid);
        // f(place, first element, keys, values) for every piece there is
        const auto walk = [&](auto f) __attribute__((always_inline)) {
            for (uint32_t i = tid; i < pieces; i += 256 * kAhead) {
                Eight<T> k[kAhead], v[kAhead];
                int32_t place[kAhead];
                uint32_t d[kAhead];
#pragma unroll
                for (uint32_t e = 0; e < kAhead; ++e) {
                    const uint32_t at = i + 256 * e;
                    place[e] = (int32_t)(at / eights);
                    d[e] = at % eights * 8;
                    if (at >= pieces || place[e] < lo || place[e] >= hi) { place[e] = -1; continue; }
                    const int64_t r = row0 + base + place[e];
                    k[e].load(k_rows + r * w.a.k_stride + d[e]);
                    v[e].load(v_rows + r * w.a.v_stride + d[e]);
                }
#pragma unroll
                for (uint32_t e = 0; e < kAhead; ++e) if (place[e] >= 0) f(place[e], d[e], k[e], v[e]);
            }
        };
        if constexpr (kNarrow) {
            // (the rows are read again behind their scales, from the caches)
            for (uint32_t i = tid; i < 2 * kPlaces; i += 256) most[0][i] = 0;
            __syncthreads();
            walk([&](int32_t place, uint32_t, const Eight<T>& k, const Eight<T>& v) { atomicMax(&most[0][place], k.most()); atomicMax(&most[1][place], v.most()); });
        }
        __syncthreads();
        walk([&](int32_t place, uint32_t d, const Eight<T>& k, const Eight<T>& v) {
            const int32_t page = pages[place / 16];
            C* ko = (C*)c.k + w.a.layer * c.layer_stride + (uint64_t)max(page, 0) * c.page_stride + ((uint64_t)h * c.page_tokens + (uint32_t)(base + place) % c.page_tokens) * D + d;
            if constexpr (kNarrow) {
                const float kf = to_scale(scale_for(__builtin_bit_cast(float, most[0][place]))), vf = to_scale(scale_for(__builtin_bit_cast(float, most[1][place])));
                if (page >= 0) *(u32x2*)ko = k.narrow(kf);
                *(u32x2*)(tile + place * row + d) = v.narrow(vf);
            } else {
                if (page >= 0) k.store(ko);
                v.store(tile + place * row + d);
            }
        });
        __syncthreads();
        // a thread to kEach places of a feature: all there are 16 bytes, some are written one by one
        constexpr uint32_t kChunks = kPlaces / kEach;
        for (uint32_t i = tid; i < kChunks * D; i += 256) {
            const uint32_t chunk = i % kChunks, d = i / kChunks;
            const int32_t from = (int32_t)(chunk * kEach), page = pages[from / 16];
            if (page < 0 || from >= hi || from + (int32_t)kEach <= lo) continue;
            C* vo = (C*)c.v + w.a.layer * c.layer_stride + page * c.page_stride + ((uint64_t)h * D + d) * c.page_tokens + (uint32_t)(base + from) % c.page_tokens;
            if (from >= lo && from + (int32_t)kEach <= hi) {
                u32x4 out{0, 0, 0, 0};
#pragma unroll
                for (uint32_t e = 0; e < kEach; ++e) {
                    if constexpr (sizeof(C) == 4) out[e] = __builtin_bit_cast(uint32_t, tile[(from + e) * row + d]);
                    else if constexpr (sizeof(C) == 2) out[e / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, tile[(from + e) * row + d]) << (16 * (e % 2));
                    else out[e / 4] |= (uint32_t)tile[(from + e) * row + d] << (8 * (e % 4));
                }
                *(u32x4*)vo = out;
            } else {
                for (uint32_t e = 0; e < kEach; ++e)
                    if (from + (int32_t)e >= lo && from + (int32_t)e < hi) vo[e] = tile[(from + e) * row + d];
            }
        }
        if constexpr (kNarrow)
            for (uint32_t i = tid; i < 2 * kPlaces; i += 256) {
                const int32_t place = (int32_t)(i % kPlaces), page = place >= lo && place < hi ? pages[place / 16] : -1;
                if (page >= 0) (i < kPlaces ? c.k_scales : c.v_scales)[w.a.layer * c.scales_layer_stride + page * c.scales_page_stride + h * c.page_tokens + (uint32_t)(base + place) % c.page_tokens] =
                    (uint8_t)scale_for(__builtin_bit_cast(float, most[i / kPlaces][place]));
            }
        __syncthreads();
    }
}

template <typename T, typename C>
hipError_t go(const KvWriteArgs& w, hipStream_t s)
{
    // (64 sequences, eight heads of 128, us of the two: of 8 tokens bf16 6.1 / 7.6, in 8 bits 6.6 / 8.2; of 16 8.6 / 8.3 and 9.2 / 11.2; of 32 14.1 / 10.0 and 15.0 / 13.0; of 500 fp32 tokens 240 / 115)
    if (w.b.max_new < (sizeof(C) == 1 ? 24u : 16u)) return launch(kv_write_kernel<T, C>, dim3(w.b.n_seqs, w.b.max_new, (w.c.heads + 3) / 4), 256, 0, s, w);
    constexpr uint32_t places = places_of<C>();
    const uint32_t groups = (uint32_t)std::min<uint64_t>(((uint64_t)w.b.max_new + places - 2) / places + 1, 4096);
    return launch(kv_write_many_kernel<T, C>, dim3(w.b.n_seqs * w.c.heads, groups), 256, places * (w.c.head_dim + (sizeof(C) == 4 ? 4 : 8)) * sizeof(C), s, w);
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& w, hipStream_t s)
{
    const bool narrow = w.c.dtype == MT_KV8;
    if (w.a.dtype == MT_BF16) return narrow ? go<__bf16, uint8_t>(w, s) : go<__bf16, __bf16>(w, s);
    return narrow ? go<float, uint8_t>(w, s) : go<float, float>(w, s);
}

}  // namespace mt
